// A decode step over the paged 8-bit cache on the 8-bit matrix instructions (bf16 layers, d_k 64 or 128).
//
// The codes go into the MFMAs as they lie in memory: nothing of K, K_LR or V is converted.  What makes that exact enough is
// that a decode step has few rows (the query heads of a key/value head) where an MFMA has sixteen: the 16-bit operand
// takes the spare rows.  A query, or a row of probabilities, is cut into three 8-bit pieces,
//   whole numbers  X = 2^16 d0 + 2^8 d1 + d2   (X = the value in units of 2^-22 of the row's largest power of two)
//   e4m3           y = p0 + 2^-4 p1 + 2^-8 p2   (each piece the nearest e4m3 number to what is left)
// and rows 4 piece + head of one 16x16x32 MFMA hold the pieces of four heads: the sum over pieces is three multiply-adds.
// Products of codes are exact in the accumulators.
//
// A page (64 tokens) of a head is one step of a wave.  Lane (n, g) = (lane % 16, lane / 16):
//   scores  A = keys: row m of the MFMA (u, parity) is token 16 (m / 4) + 8 u + 2 (m % 4) + parity, so that lane (n, g) ends with
//           tokens 16 g .. 16 g + 15 of column n; B = the query's pieces in columns 4 piece + head; summed over the pieces
//           (rotations inside the 16 lanes) every lane has the scores of head n % 4;
//   P V     A = pieces of the probabilities: lane (n, g) makes piece n / 4 of what it has itself, no lane moves; B = V: 16 bytes of a
//           lane are tokens 16 g .. 16 g + 15 of feature n; D row 4 g + v: piece g of head v.
#pragma once
#include "kernels_cache8.h"
#include "kernels_prefill.h"
#include "mfma_ffn.h"

namespace lisa {

typedef int c8_i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int c8_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long c8_u64_a2 __attribute__((aligned(2)));

constexpr int C8_NO_QUERY = 1 << 20;   // exponent of a row with an infinity or a NaN: its scores are NaN
template <int FMT> struct mfma8;
template <> struct mfma8<0> {
  typedef c8_i32x4 acc;
  static __device__ __forceinline__ acc zero() { return acc{0, 0, 0, 0}; }
  static __device__ __forceinline__ acc mul(unsigned long long a, unsigned long long b, acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x32_i8((long)a, (long)b, c, 0, 0, 0);
  }
  // weight of piece p of a query of which 2^e is the largest power of two; of a probability
  static __device__ __forceinline__ float query_weight(int p, int e) { return e == C8_NO_QUERY ? NAN : ldexpf(1.f, e - 5 - 8 * p); }
  static __device__ __forceinline__ float prob_weight(int p) { return p == 0 ? 0x1p-6f : p == 1 ? 0x1p-14f : 0x1p-22f; }
};
template <> struct mfma8<1> {
  typedef f32x4 acc;
  static __device__ __forceinline__ acc zero() { return acc{0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ acc mul(unsigned long long a, unsigned long long b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8((long)a, (long)b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ float query_weight(int p, int e) { return e == C8_NO_QUERY ? NAN : ldexpf(1.f, e - 7 - 4 * p); }
  static __device__ __forceinline__ float prob_weight(int p) { return p == 0 ? 0x1p-8f : p == 1 ? 0x1p-12f : 0x1p-16f; }
};

__device__ __forceinline__ unsigned fp8_pack(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Four elements of a query, |x| < 2^(e + 1), as their three pieces.
template <int FMT>
__device__ __forceinline__ void query_pieces(const float (&x)[4], int e, unsigned (&w)[3]) {
  if constexpr (FMT == 0) {
    unsigned X[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) X[i] = (unsigned)((int)rintf(ldexpf(x[i], 21 - e)) + 0x8080);   // |X| <= 2^22; d1, d2 carry 128
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      w[p] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[p] |= (X[i] >> (16 - 8 * p) & 0xffu) << (8 * i);
    }
    w[1] ^= 0x80808080u, w[2] ^= 0x80808080u;
  } else {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = ldexpf(x[i], 7 - e);
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      w[p] = fp8_pack(y[0], y[1], y[2], y[3]);
      y[0] = (y[0] - __builtin_amdgcn_cvt_f32_fp8((int)w[p], 0)) * 16.f;
      y[1] = (y[1] - __builtin_amdgcn_cvt_f32_fp8((int)w[p], 1)) * 16.f;
      y[2] = (y[2] - __builtin_amdgcn_cvt_f32_fp8((int)w[p], 2)) * 16.f;
      y[3] = (y[3] - __builtin_amdgcn_cvt_f32_fp8((int)w[p], 3)) * 16.f;
    }
  }
}
// The pieces of H rows of n <= W elements in the LDS, codes [h][piece][W], exps [h], by all threads of the workgroup
// (W / 4 lanes, at most 64, per row).  src(h): the row.  load() issues the loads of the first rows; what is loaded between it and
// store() does not have to arrive for them.
template <int FMT, int W>
__device__ __forceinline__ void store_query(const unsigned short (&raw)[4], int h, int l, int H, int n, unsigned char* codes, int* exps) {
  constexpr int LPR = W / 4;
  float x[4], m = 0.f;
  int bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = 4 * l + i < n ? bf16_bits_to_f32(raw[i]) : 0.f;
    bad |= !(fabsf(x[i]) < INFINITY);
    m = fmaxf(m, fabsf(x[i]));
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor(m, o, 64));
    bad |= __shfl_xor(bad, o, 64);
  }
  const int e = m > 0.f && !bad ? __builtin_amdgcn_frexp_expf(m) - 1 : 0;
  unsigned w[3];
  query_pieces<FMT>(x, e, w);
  if (h < H) {
#pragma unroll
    for (int p = 0; p < 3; ++p) *(unsigned*)(codes + (h * 3 + p) * W + 4 * l) = w[p];
    if (l == 0) exps[h] = bad ? C8_NO_QUERY : e;
  }
}
template <int W>
struct QueryStage {
  static constexpr int LPR = W / 4;                          // lanes per row (a power of two)
  static_assert(LPR <= 64 && (LPR & (LPR - 1)) == 0, "lanes per row");
  unsigned short raw[4];
  template <class Src>
  __device__ __forceinline__ void load(int e0, int H, int n, int tid, Src&& src) {
    const bf16_t* q = src(min((e0 + tid) / LPR, H - 1));
    const int l = tid % LPR;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = q[min(4 * l + i, n - 1)].bits;
  }
  template <class Src>
  __device__ __forceinline__ void store(bool e4m3, int H, int n, unsigned char* codes, int* exps, int tid, int nthreads, Src&& src) {
    for (int e0 = 0; e0 < H * LPR; e0 += nthreads) {         // (nthreads is a multiple of LPR: whole rows)
      if (e0) load(e0, H, n, tid, src);
      if (e4m3) store_query<1, W>(raw, (e0 + tid) / LPR, tid % LPR, H, n, codes, exps);
      else store_query<0, W>(raw, (e0 + tid) / LPR, tid % LPR, H, n, codes, exps);
    }
  }
};

// Scores of a page against the four heads of a tile: x[f] = score of token 16 g + f, head n % 4.
// kreg[s][u]: 16 bytes of a lane, tokens T and T + 1 (T = 16 (n / 4) + 8 u + 2 (n % 4)), features 32 s + 8 g .. + 7.  page_products may be
// called for several key blocks, with zeros in the columns of the heads that do not go with them.
template <int FMT, int KS>
__device__ __forceinline__ void page_products(const c8_u32x4 (&kreg)[KS][2], const unsigned long long (&qc)[KS], typename mfma8<FMT>::acc (&acc)[2][2]) {
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      acc[u][0] = mfma8<FMT>::mul(kreg[s][u][0] | (unsigned long long)kreg[s][u][1] << 32, qc[s], acc[u][0]);
      acc[u][1] = mfma8<FMT>::mul(kreg[s][u][2] | (unsigned long long)kreg[s][u][3] << 32, qc[s], acc[u][1]);
    }
}
// weight: of this lane's piece, with the scales.
template <int FMT>
__device__ __forceinline__ void page_sums(const typename mfma8<FMT>::acc (&acc)[2][2], float weight, float (&x)[16]) {
#pragma unroll
  for (int f = 0; f < 16; ++f) {
    x[f] = (float)acc[f >> 3][f & 1][(f & 7) >> 1] * weight;
    x[f] += dpp_move<0x128>(x[f]);                           // row_ror:8
    x[f] += dpp_move<0x124>(x[f]);                           // row_ror:4
  }
}
// The four of sixteen values that quarter `pc` of the lanes keeps.  (The values are pinned: else the choice becomes branches around what
// they are made of.)
__device__ __forceinline__ void quarter(float (&x)[16], int pc, float (&y)[4]) {
#pragma unroll
  for (int f = 0; f < 16; ++f) asm volatile("" : "+v"(x[f]));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = pc & 1 ? x[4 + i] : x[i], hi = pc & 1 ? x[12 + i] : x[8 + i];
    y[i] = pc & 2 ? hi : lo;
  }
}
__device__ __forceinline__ int page_token(int n, int u) { return 16 * (n >> 2) + 8 * u + 2 * (n & 3); }

// Piece `pc` (0 .. 2; 3: zeros) of 16 probabilities as MFMA operands.
template <int FMT>
__device__ __forceinline__ void prob_pieces(const float (&p)[16], int pc, unsigned long long (&op)[2]) {
  unsigned w[4];
  if constexpr (FMT == 0) {
    // the low bits of p 2^22 + 2^23 + 0x8080 are X + 0x8080, X = p 2^22 rounded: byte 2 is d0, bytes 1 and 0 are d1 + 128, d2 + 128
    const unsigned sel = pc == 3 ? 0x0c0c0c0cu : pc == 0 ? 0x0c0c0602u : pc == 1 ? 0x0c0c0501u : 0x0c0c0400u;
    const unsigned flip = pc == 1 || pc == 2 ? 0x80808080u : 0u;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      unsigned y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = __float_as_uint(__builtin_fmaf(p[4 * q + i], 4194304.f, 8388608.f + 32896.f));
      const unsigned lo = __builtin_amdgcn_perm(y[1], y[0], sel), hi = __builtin_amdgcn_perm(y[3], y[2], sel);
      w[q] = (lo | hi << 16) ^ flip;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = p[4 * q + i] * 256.f;
      unsigned c[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        c[k] = fp8_pack(y[0], y[1], y[2], y[3]);
        if (k == 2) break;
        y[0] = (y[0] - __builtin_amdgcn_cvt_f32_fp8((int)c[k], 0)) * 16.f;
        y[1] = (y[1] - __builtin_amdgcn_cvt_f32_fp8((int)c[k], 1)) * 16.f;
        y[2] = (y[2] - __builtin_amdgcn_cvt_f32_fp8((int)c[k], 2)) * 16.f;
        y[3] = (y[3] - __builtin_amdgcn_cvt_f32_fp8((int)c[k], 3)) * 16.f;
      }
      w[q] = pc & 2 ? (pc & 1 ? 0u : c[2]) : pc & 1 ? c[1] : c[0];
    }
  }
  op[0] = w[0] | (unsigned long long)w[1] << 32;
  op[1] = w[2] | (unsigned long long)w[3] << 32;
}

// Reductions over g (lanes n, n + 16, n + 32, n + 48), the result in all four.
template <class Op>
__device__ __forceinline__ float groups_reduce(float v, Op op) {
  const unsigned u = __float_as_uint(v);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const unsigned w = __float_as_uint(v);
  auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return op(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

__device__ __forceinline__ c8_u32x4 c8_stream(const unsigned char* p) { return __builtin_nontemporal_load((const c8_u32x4*)p); }

// ---- scores of a LiSA layer -----------------------------------------------------------------------
struct Cache8ScoresArgs {
  Cache8View c;
  const bf16_t* q;            // [B,H,w]
  const half_t* prev;         // [B,H,Lk]
  const bf16_t* w1;           // [Din,F]
  const bf16_t* w2;           // [F,H]; null: a single layer (w1 is [Din,H], F = 2 H)
  half_t* row;                // [B,H,Lk] or null
  float* s;                   // A_n, [B][pages][H][64]
  int H, Lk, Lp, F, fmt;
  int n_pages;                // pages per workgroup, at most 64
  float scale;
};
constexpr int C8_SROW = PG_TOK + 4;                          // floats per head of the a_delta tile
constexpr int cache8_scores_lds(int H, int ks, int w_bytes) {   // (a row more per tile: what lies past the heads)
  return (2 * (H + 1) * C8_SROW + (H + 3) / 4 * 4) * 4 + H * 3 * 32 * ks + w_bytes;
}

// The image of MfmaFfn::stage() by 256 threads.  Rows of even length: a thread takes eight rows of two columns, which are two 16-byte pieces of
// the image; load() issues all loads (ahead of the first page's), store() puts them in place.  (64 -> 256 -> 32, 8 x 2500 tokens: 31 us for the launch with
// 16-byte loads along the rows, whose elements go to LDS banks that collide; 19 with a launch in front that makes the image.)  w2 null:
// y = w1^T x as the ReLU network [w1, -w1], [I; -I].
template <int KS, int FS, int HBO>
struct FfnStage {
  static constexpr int T1 = KS * 4 * 16 * FS, T2 = FS * 4 * 8 * HBO;   // (k-step, g, column pair)
  static constexpr int N1 = (T1 + 255) / 256, N2 = (T2 + 255) / 256;
  unsigned x1[N1][8], x2[N2][8];
  static __device__ __forceinline__ bool pairs(const Cache8ScoresArgs& a) { return a.w2 && a.F % 2 == 0 && a.H % 2 == 0; }
  __device__ __forceinline__ void load(const Cache8ScoresArgs& a, int Din, int tid) {
    if (!pairs(a)) return;
#pragma unroll
    for (int i = 0; i < N1; ++i) {
      const int e = min(tid + 256 * i, T1 - 1), f = 2 * (e % (16 * FS)), r = e / (16 * FS) * 8;   // rows r .. r + 7
#pragma unroll
      for (int k = 0; k < 8; ++k) x1[i][k] = *(const unsigned*)(a.w1 + (unsigned)min(r + k, Din - 1) * a.F + min(f, a.F - 2));
    }
#pragma unroll
    for (int i = 0; i < N2; ++i) {
      const int e = min(tid + 256 * i, T2 - 1), h = 2 * (e % (8 * HBO)), o = e / (8 * HBO), r = 32 * (o >> 2) + 4 * (o & 3);
#pragma unroll
      for (int k = 0; k < 8; ++k) x2[i][k] = *(const unsigned*)(a.w2 + (unsigned)min(r + 16 * (k >> 2) + (k & 3), a.F - 1) * a.H + min(h, a.H - 2));
    }
  }
  __device__ __forceinline__ static unsigned short* at1(unsigned short* lds, int ch, int f) {
    return lds + (((f >> 4) * KS + (ch >> 5)) * 64 + (ch >> 3 & 3) * 16 + (f & 15)) * 8 + (ch & 7);
  }
  __device__ __forceinline__ static unsigned short* at2(unsigned short* lds, int f, int h) {
    const int r = f & 31;
    return lds + 2 * FS * KS * 512 + (((h >> 4) * FS + (f >> 5)) * 64 + (r >> 2 & 3) * 16 + (h & 15)) * 8 + 4 * (r >> 4) + (r & 3);
  }
  // the low (high) halves of eight pairs, as halves, zero where `in` says so
  template <class In>
  __device__ __forceinline__ static u16x8 piece(const unsigned (&x)[8], int high, In&& in) {
    u16x8 v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = in(k) ? half_bits(high ? __uint_as_float(x[k] & 0xffff0000u) : bf16_bits_to_f32(x[k] & 0xffffu)) : (unsigned short)0;
    return v;
  }
  __device__ __forceinline__ void store(const Cache8ScoresArgs& a, int Din, unsigned short* lds, int tid) {
    if (pairs(a)) {
#pragma unroll
      for (int i = 0; i < N1; ++i) {
        const int e = tid + 256 * i, f = 2 * (e % (16 * FS)), r = e / (16 * FS) * 8;
        if (e < T1)
#pragma unroll
          for (int c = 0; c < 2; ++c) *(u16x8*)at1(lds, r, f + c) = piece(x1[i], c, [&](int k) { return r + k < Din && f < a.F; });
      }
#pragma unroll
      for (int i = 0; i < N2; ++i) {
        const int e = tid + 256 * i, h = 2 * (e % (8 * HBO)), o = e / (8 * HBO), r = 32 * (o >> 2) + 4 * (o & 3);
        if (e < T2)
#pragma unroll
          for (int c = 0; c < 2; ++c) *(u16x8*)at2(lds, r, h + c) = piece(x2[i], c, [&](int k) { return r + 16 * (k >> 2) + (k & 3) < a.F && h < a.H; });
      }
      return;
    }
    const int H = a.H, cols = a.w2 ? a.F : H;
#pragma unroll 4
    for (int e = tid; e < 32 * KS * 32 * FS; e += 256) {
      const int ch = e / (32 * FS), f = e % (32 * FS);
      const unsigned v = a.w1[(size_t)min(ch, Din - 1) * cols + min(f < cols ? f : f - cols, cols - 1)].bits;
      const float y = bf16_bits_to_f32(v);
      *at1(lds, ch, f) = ch < Din && f < a.F ? half_bits(f < cols ? y : -y) : (unsigned short)0;
    }
#pragma unroll 4
    for (int e = tid; e < 32 * FS * 16 * HBO; e += 256) {
      const int f = e / (16 * HBO), h = e % (16 * HBO);
      float y = f == h ? 1.f : f == H + h ? -1.f : 0.f;
      if (a.w2) y = bf16_bits_to_f32(a.w2[(size_t)min(f, a.F - 1) * H + min(h, H - 1)].bits);
      *at2(lds, f, h) = f < a.F && h < H ? half_bits(y) : (unsigned short)0;
    }
  }
};

// The FFN of sixteen tokens from the image of MfmaFfn::stage().  What is not a half number already, A_delta and the hidden units, goes in as two (x and what
// is left of it, 2^-22 together): rounded to one half each, these add as much to a row's error as the half number that it is handed on in.
// 32 hidden units at a time; the weights of the next 32 are read while these are multiplied.
template <int ACT, int KX, int FS, int HBO, bool LO>
__device__ __forceinline__ void cache8_ffn(const unsigned short* lds, const f16x8 (&x)[KX], const f16x8 (&xl)[LO ? KX : 1], f32x4 (&y)[HBO]) {
  const int lane = threadIdx.x & 63;
  const unsigned short* l1 = lds + lane * 8;
  const unsigned short* l2 = l1 + 2 * FS * KX * 512;
  f16x8 w1[2][2][KX], w2[2][HBO];
  auto read = [&](int s, f16x8 (&a)[2][KX], f16x8 (&b)[HBO]) {
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int ks = 0; ks < KX; ++ks) a[half][ks] = *(const f16x8*)(l1 + ((2 * s + half) * KX + ks) * 512);
#pragma unroll
    for (int hb = 0; hb < HBO; ++hb) b[hb] = *(const f16x8*)(l2 + (hb * FS + s) * 512);
  };
  read(0, w1[0], w2[0]);
#pragma unroll
  for (int hb = 0; hb < HBO; ++hb) y[hb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < FS; ++s) {
    if (s + 1 < FS) read(s + 1, w1[(s + 1) & 1], w2[(s + 1) & 1]);
    f16x8 hi, lo;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KX; ++ks) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(w1[s & 1][half][ks], x[ks], acc, 0, 0, 0);
        if (LO) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(w1[s & 1][half][ks], xl[LO ? ks : 0], acc, 0, 0, 0);
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float u = acc[v];
        if (ACT == 1) {                                      // (exp2 of a very negative u: inf, 1 / inf = 0)
          u = fminf(u * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u)), 65504.f);
        } else {
          u = __builtin_amdgcn_fmed3f(u, 0.f, 65504.f);
        }
        hi[4 * half + v] = (half_t)u;
        lo[4 * half + v] = (half_t)(u - (float)hi[4 * half + v]);
      }
    }
#pragma unroll
    for (int hb = 0; hb < HBO; ++hb) {
      y[hb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w2[s & 1][hb], hi, y[hb], 0, 0, 0);
      y[hb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w2[s & 1][hb], lo, y[hb], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// MODE 0: A_n = A_{n-1} + A_delta, 1: FFN(A_{n-1}) + A_delta, 2: FFN([A_{n-1}; A_delta]).  KS: pieces of 32 features of a K_LR row.
// grid (ceil(pages / n_pages), B), block 256: n_pages pages of a sequence, all heads.  Per page the waves take tiles of four heads in turn
// (A_delta to the LDS), then 16 tokens each through the FFN; the next page's keys and A_{n-1} are loaded where this one's have been used, and one
// barrier a page (two A_delta tiles) lets the waves run apart.  float32 A_n to `s` for k_cache8_pv.
// KVT: key/value heads that the four heads of a tile can have, 1 (groups of whole tiles) or 4; their products go into one accumulator, so that what
// follows on the vector ALU (16 sums over the pieces) is done once per tile.
// Bound: the chain of a page (products, sums over the pieces, LDS, FFN, LDS) on two waves per SIMD, some 540 vector instructions per
// page and wave, with the next page's loads under way: 57 us for the 215 MB of 64 sequences of up to 4097 tokens, 32 heads (3.8 TB/s).
template <int HBI, int FS, int HBO, int ACT, int MODE, int KS, int KVT>
__global__ __launch_bounds__(256, 2) void k_cache8_scores_mfma(Cache8ScoresArgs a) {
  typedef MfmaFfn<HBI, FS, HBO, ACT> Ffn;
  constexpr int KX = MODE == 0 ? 1 : Ffn::KS, KP = MODE == 2 ? (KX + 1) / 2 : KX;   // pieces of 32 channels, those with A_{n-1}
  extern __shared__ __align__(16) float c8_lds[];
  const Cache8View& c = a.c;
  const int H = a.H, Din = MODE == 2 ? 2 * H : H;
  float* a_s = c8_lds;                                       // [2][H + 1][C8_SROW]
  int* e_s = (int*)(a_s + 2 * (H + 1) * C8_SROW);            // [H]
  unsigned char* q_s = (unsigned char*)(e_s + (H + 3) / 4 * 4);   // [H][3][32 KS]
  unsigned short* w_s = (unsigned short*)(q_s + H * 3 * 32 * KS);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col0 = blockIdx.x * a.n_pages, b = blockIdx.y;
  const int my_col = col0 + lane;                            // lane i: the workgroup's page i
  const int entry = c.entry(b, my_col), len = min(c.lens[b], a.Lk);
  const int id = lane < a.n_pages && (long long)my_col * PG_TOK < len ? entry : -1;
  unsigned long long todo = __ballot(id >= 0);
  if (!todo) return;
  const int n = lane & 15, g = lane >> 4;
  const int pj = 16 * wv + n;                                // this lane's token in the FFN
  const int group = H / c.Hkv, tiles = (H + 3) / 4;
  const int hn = n & 3, pc = n >> 2;
  // keys: the tiles of this wave, UN of them in flight
  constexpr int UN = KVT == 4 || KS == 2 ? 1 : 2;            // (two tiles of four key/value heads do not fit the register file)
  const int np = c.w8 / 8;
  const int rounds = (tiles + 4 * UN - 1) / (4 * UN);        // of UN tiles per wave and page (past the last tile: the last one again)
  unsigned k_at[KS];                                         // this lane's place in a block of keys
#pragma unroll
  for (int s = 0; s < KS; ++s) k_at[s] = (min(4 * s + g, np - 1) * PG_TOK + page_token(n, 0)) * 8;
  struct Tile {
    c8_u32x4 k[KVT][KS][2];
    float scale;                                             // of this lane's head
  };
  Tile in[UN];
  auto load_k = [&](int page, int tile, Tile& t) {
    tile = min(tile, tiles - 1);
    const int kv0 = 4 * tile / group, kv1 = min(4 * tile + 3, H - 1) / group;
    t.scale = c.k_scale[(size_t)page * c.Hkv + min(4 * tile + hn, H - 1) / group];
#pragma unroll
    for (int v = 0; v < KVT; ++v) {
      const unsigned char* kb = c.k_block(page, min(kv0 + v, kv1));
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u) t.k[v][s][u] = c8_stream(kb + k_at[s] + u * 64);
    }
  };
  // A_{n-1} of this lane's token: what the FFN takes (clamped; past the heads and the end it is zeroed where it is used).  One element per
  // register: to pack them is to wait for them.
  unsigned short xin[KP][8];
  auto load_x = [&](int i) {
    const unsigned short* xp = (const unsigned short*)a.prev + (size_t)b * H * a.Lk;   // (32-bit offsets: H Lk < 2^30)
    const unsigned j = min((col0 + i) * PG_TOK + pj, len - 1);
    if (MODE != 0)
#pragma unroll
      for (int ks = 0; ks < KP; ++ks)
#pragma unroll
        for (int e = 0; e < 8; ++e) xin[ks][e] = xp[(unsigned)min(32 * ks + 8 * g + e, H - 1) * (unsigned)a.Lk + j];
  };
  auto src = [&](int h) { return a.q + ((size_t)b * H + h) * c.w; };
  QueryStage<32 * KS> qst;
  qst.load(0, H, c.w, tid, src);
  FfnStage<KX, FS, HBO> fst;
  if (MODE != 0) fst.load(a, Din, tid);
  int at = __builtin_ctzll(todo), buf = 0;
  {
    const int page = __builtin_amdgcn_readlane(id, at);
#pragma unroll
    for (int i = 0; i < UN; ++i) load_k(page, wv + 4 * i, in[i]);
    load_x(at);
  }
  qst.store(a.fmt, H, c.w, q_s, e_s, tid, 256, src);
  if (MODE != 0) fst.store(a, Din, w_s, tid);
  lds_barrier();
  auto delta = [&](auto fmt, int tile, const Tile& t, float* to) __attribute__((always_inline)) {
    constexpr int FMT = decltype(fmt)::value;
    typedef mfma8<FMT> M;
    const int h = min(4 * tile + hn, H - 1), mine = h / group, kv0 = 4 * tile / group;
    unsigned long long qc[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qc[s] = *(const unsigned long long*)(q_s + (h * 3 + min(pc, 2)) * (32 * KS) + 32 * s + 8 * g);
      if (pc == 3) qc[s] = 0;
    }
    typename M::acc acc[2][2] = {{M::zero(), M::zero()}, {M::zero(), M::zero()}};
#pragma unroll
    for (int v = 0; v < KVT; ++v) {
      unsigned long long qv[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) qv[s] = KVT == 1 || mine == kv0 + v ? qc[s] : 0;
      page_products<FMT, KS>(t.k[v], qv, acc);
    }
    float xs[16];
    page_sums<FMT>(acc, M::query_weight(pc, e_s[h]) * (t.scale * a.scale), xs);
    float y[4];
    quarter(xs, pc, y);
    if (4 * tile + hn < H) {                                 // lane (head, quarter, g): four of its sixteen tokens
      *(f32x4*)(to + h * C8_SROW + 16 * g + 4 * pc) = f32x4{y[0], y[1], y[2], y[3]};
    }
  };
  auto step = [&](int next, auto more) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more)::value;
    const int page = __builtin_amdgcn_readlane(id, at), page_n = MORE ? __builtin_amdgcn_readlane(id, next) : 0;
    float* to = a_s + buf * (H + 1) * C8_SROW;
    auto tile_of = [&](int r, int i) { return wv + 4 * (r * UN + i); };
    auto use = [&](int r, int i) __attribute__((always_inline)) {
      if (tile_of(r, i) >= tiles) return;
      if (a.fmt) delta(std::integral_constant<int, 1>{}, tile_of(r, i), in[i], to);
      else delta(std::integral_constant<int, 0>{}, tile_of(r, i), in[i], to);
    };
    for (int r = 0; r + 1 < rounds; ++r)
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        use(r, i);
        load_k(page, tile_of(r + 1, i), in[i]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
    for (int i = 0; i < UN; ++i) {                           // (no branch around these loads: what comes after them waits for older ones only)
      use(rounds - 1, i);
      if (MORE) load_k(page_n, tile_of(0, i), in[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    lds_barrier();
    // A_n of sixteen tokens of a wave's: lane -> head (16 of them at a time), four tokens
    const int t_out = 16 * wv + 4 * (lane & 3), j_out = (col0 + at) * PG_TOK + t_out, h_out = lane >> 2;
    float* sp = a.s + ((size_t)b * (a.Lp / PG_TOK) + col0 + at) * H * PG_TOK + t_out;
    half_t* rp = a.row ? a.row + (size_t)b * H * a.Lk + j_out : nullptr;
    auto emit = [&](int h, const f32x4& y) __attribute__((always_inline)) {
      *(f32x4*)(sp + h * PG_TOK) = y;
      if (!rp) return;
      half_t* r = rp + (size_t)h * a.Lk;
      typedef _Float16 f16x4_ __attribute__((ext_vector_type(4)));
      const f16x4_ v = {f32_to_half_sat(y[0]), f32_to_half_sat(y[1]), f32_to_half_sat(y[2]), f32_to_half_sat(y[3])};
      if (MORE || j_out + 4 <= len) {                        // (a page with another one behind it is full)
        *(c8_u64_a2*)r = __builtin_bit_cast(unsigned long long, v);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j_out + i < len) r[i] = v[i];
      }
    };
    if constexpr (MODE == 0) {
      for (int h = h_out; h < H; h += 16) {
        f32x4 y = *(const f32x4*)(to + h * C8_SROW + t_out);
        const half_t* xp = a.prev + ((size_t)b * H + h) * a.Lk;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += (float)xp[min(j_out + i, len - 1)];
        emit(h, y);
      }
    } else {
      // (what follows from the lane's number is made anew: kept over the pages, it does not fit the registers)
      int go = g, po = pj;
      asm volatile("" : "+v"(go), "+v"(po));
      f16x8 x[KX], xl[MODE == 2 ? KX : 1];
#pragma unroll
      for (int ks = 0; ks < KX; ++ks)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int ch = 32 * ks + 8 * go + e;
          x[ks][e] = ks < KP ? __builtin_bit_cast(half_t, xin[ks < KP ? ks : 0][e]) : (_Float16)0.f;
          if constexpr (MODE == 2) {
            float u = 0.f;
            if (ch >= H) {
              u = ch < Din ? to[(ch - H) * C8_SROW + po] : 0.f;
              x[ks][e] = f32_to_half_sat(u);
              u -= (float)x[ks][e];
            }
            xl[ks][e] = f32_to_half_sat(u);
          } else if (ch >= Din) {
            x[ks][e] = (_Float16)0.f;
          }
        }
      if (MORE) load_x(next);
      f32x4 y[HBO];
      cache8_ffn<ACT, KX, FS, HBO, MODE == 2>(w_s, x, xl, y);
      // this wave's tokens of the tile become A_n (no other wave has business with them), and go out as rows
      float d[HBO][4];
#pragma unroll
      for (int hb = 0; hb < HBO; ++hb)
#pragma unroll
        for (int v = 0; v < 4; ++v) d[hb][v] = MODE == 2 ? 0.f : to[min(16 * hb + 4 * go + v, H) * C8_SROW + po];
#pragma unroll
      for (int hb = 0; hb < HBO; ++hb)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          to[min(16 * hb + 4 * go + v, H) * C8_SROW + po] = y[hb][v] + d[hb][v];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int hb = 0; hb < HBO; ++hb)
        if (16 * hb + h_out < H) emit(16 * hb + h_out, *(const f32x4*)(to + (16 * hb + h_out) * C8_SROW + t_out));
    }
    buf ^= 1;
  };
  todo &= todo - 1;
  while (todo) {
    const int next = __builtin_ctzll(todo);
    todo &= todo - 1;
    step(next, std::true_type{});
    at = next;
  }
  step(0, std::false_type{});
}

// ---- softmax and P V --------------------------------------------------------------------------------
struct Cache8PvArgs {
  Cache8View c;
  const bf16_t* q;        // MODE 0: [B,H,DK]
  const float* s;         // MODE 1: A_n [B][pages][H][64]
  const half_t* prev;     // MODE 2: A_n [B,H,Lk]
  half_t* row;            // MODE 0, 2: A_n out [B,H,Lk] or null
  void* out;              // [B,H,d_k]
  float* part_o;          // [B][n_span][H][d_k]   (n_span > 1)
  float* part_ml;         // [B][n_span][H][2]
  int H, Lk, Lp, n_span, span_pages, out_f32;
  int chunks;             // workgroups that the query heads of a key/value head are dealt to, 4 GT each
  int f_parts;            // MODE 1, 2: workgroups that its features are dealt to, DK each
  float scale;
};

// MODE 0: a standard layer (scores from K), 1: scores given in float32, 2: in half, emitted as they are.
// DK: features of a workgroup (MODE 0: d_k).
// grid (Hkv chunks f_parts, n_span, B), block 64 NW: the pages of a span are dealt to the waves, each with softmax state and sums of its own,
// merged through the LDS at the end; spans by k_cache8_combine.  Bound: the stream of K and V (a page of a head is loaded where the
// one before it has been used, so that every wave has loads in flight; 64 sequences of up to 4097 tokens, 32 heads: 132 us, 6.6 TB/s; standard,
// 32 of 8192, 8 kv heads: 425 MB in 75 us, 5.7 TB/s, 92 us with the score rows, whose stores cost the same in front of the loads, behind them, and
// non-temporal); the vector ALU needs 150 - 220 instructions for the
// 8 or 16 KB of a step.
// GT: tiles of four query heads, GH: heads of a tile that are there (1: one query head per key/value head).
template <int FMT, int DK, int MODE, int GT, int GH, int NW>
__global__ __launch_bounds__(64 * NW, MODE == 0 && NW == 4 && GT == 1 && GH == 1 ? 3 : 1) void k_cache8_pv(Cache8PvArgs a) {
  typedef mfma8<FMT> M;
  constexpr int KS = DK / 32, NT = DK / 16;
  constexpr float LOG2E = 1.4426950408889634f;
  __shared__ __align__(16) float o_s[NW][GT * GH][DK];
  __shared__ float ml_s[NW][GT * 4][2];
  __shared__ __align__(16) unsigned char q_s[MODE == 0 ? GT * 4 * 3 * DK : 16];
  __shared__ int e_s[GT * 4];
  const Cache8View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4, hn = n & 3, pc = n >> 2;
  const int dk = MODE == 0 ? DK : c.dk, f0 = MODE == 0 ? 0 : blockIdx.x % a.f_parts * DK;
  const int kvc = MODE == 0 ? blockIdx.x : blockIdx.x / a.f_parts;
  const int b = blockIdx.z, span = blockIdx.y, kv = kvc / a.chunks, chunk = kvc % a.chunks;
  const int group = a.H / c.Hkv, h0 = chunk * 4 * GT, heads = min(4 * GT, group - h0);   // heads of this workgroup
  const int head0 = kv * group + h0;
  // lane i: page p_begin + wv + NW i (span_pages <= 64 NW)
  const int p_begin = span * a.span_pages, my_col = p_begin + wv + NW * lane;
  const int entry = c.entry(b, my_col), len = max(min(c.lens[b], a.Lk), 0);
  const int n_pages = (len + PG_TOK - 1) / PG_TOK, p_end = min(n_pages, p_begin + a.span_pages);
  if (p_begin >= n_pages && a.n_span > 1) return;            // (k_cache8_combine knows)
  const int id = my_col < p_end ? entry : -1;
  const size_t id_at = (size_t)max(id, 0) * c.Hkv + kv;
  const float ksc = MODE == 0 ? c.k_scale[id_at] : 0.f, vsc = c.v_scale[id_at];
  unsigned long long todo = __ballot(id >= 0);

  c8_u32x4 kreg[MODE == 0 ? KS : 1][2], vreg[NT];
  float sreg[MODE == 1 ? GT : 1][16];
  half_t hreg[MODE == 2 ? GT : 1][16];
  auto load_k = [&](int i) {
    if constexpr (MODE == 0) {
      const unsigned char* kb = c.k_block(__builtin_amdgcn_readlane(id, i), kv) + page_token(n, 0) * 8 + g * (PG_TOK * 8);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u) kreg[s][u] = c8_stream(kb + s * (4 * PG_TOK * 8) + u * 64);
    }
  };
  auto load_v = [&](int i) {
    const unsigned char* vb = c.v_block(__builtin_amdgcn_readlane(id, i), kv) + (f0 + n) * PG_TOK + 16 * g;
#pragma unroll
    for (int t = 0; t < NT; ++t) vreg[t] = c8_stream(vb + t * (16 * PG_TOK));
  };
  auto load_s = [&](int i) {
    const int j = (p_begin + wv + NW * i) * PG_TOK + 16 * g;
    if constexpr (MODE == 1) {
#pragma unroll
      for (int t = 0; t < GT; ++t) {
        const float* sp = a.s + (((size_t)b * (a.Lp / PG_TOK) + p_begin + wv + NW * i) * a.H + head0 + min(4 * t + hn, heads - 1)) * PG_TOK + 16 * g;
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4*)&sreg[t][4 * q] = *(const f32x4*)(sp + 4 * q);
      }
    }
    if constexpr (MODE == 2) {
#pragma unroll
      for (int t = 0; t < GT; ++t) {
        const half_t* sp = a.prev + ((size_t)b * a.H + head0 + min(4 * t + hn, heads - 1)) * a.Lk;
#pragma unroll
        for (int f = 0; f < 16; ++f) hreg[t][f] = sp[min(j + f, len - 1)];
      }
    }
  };
  QueryStage<DK> qst;
  auto src = [&](int h) { return a.q + ((size_t)b * a.H + head0 + min(h, heads - 1)) * DK; };
  if constexpr (MODE == 0) qst.load(0, GT * 4, DK, tid, src);
  int i = todo ? __builtin_ctzll(todo) : 0;
  if (todo) {
    load_k(i);
    load_s(i);
    load_v(i);
  }
  unsigned long long qc[MODE == 0 ? GT : 1][KS];
  float qw[MODE == 0 ? GT : 1];
  if constexpr (MODE == 0) {
    qst.store(FMT == 1, GT * 4, DK, q_s, e_s, tid, 64 * NW, src);
    lds_barrier();
#pragma unroll
    for (int t = 0; t < GT; ++t) {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        qc[t][s] = *(const unsigned long long*)(q_s + ((4 * t + hn) * 3 + min(pc, 2)) * DK + 32 * s + 8 * g);
        if (pc == 3) qc[t][s] = 0;
      }
      qw[t] = M::query_weight(pc, e_s[4 * t + hn]) * a.scale;
    }
  }
  const float pw = g == 3 ? 0.f : M::prob_weight(g);
  float m_run[GT], l_run[GT], o[GT][NT][GH];
#pragma unroll
  for (int t = 0; t < GT; ++t) {
    m_run[t] = -INFINITY, l_run[t] = 0.f;
#pragma unroll
    for (int d = 0; d < NT; ++d)
#pragma unroll
      for (int v = 0; v < GH; ++v) o[t][d][v] = 0.f;
  }
  auto step = [&](int at, int next, auto more) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more)::value;
    const int col = p_begin + wv + NW * at, n_here = min(len - col * PG_TOK, PG_TOK);
    const float k_scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc), at));
    const float v_scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc), at));
    unsigned long long pop[GT][2];
    float x[GT][16];
#pragma unroll
    for (int t = 0; t < GT; ++t) {
      if constexpr (MODE == 0) {
        typename M::acc acc[2][2] = {{M::zero(), M::zero()}, {M::zero(), M::zero()}};
        page_products<FMT, KS>(kreg, qc[t], acc);
        page_sums<FMT>(acc, qw[t] * k_scale, x[t]);
      } else {
#pragma unroll
        for (int f = 0; f < 16; ++f) x[t][f] = MODE == 1 ? sreg[t][f] : (float)hreg[t][f];
      }
    }
    if constexpr (MORE) {
      load_k(next);
      load_s(next);
    }
#pragma unroll
    for (int t = 0; t < GT; ++t) {
      if (MODE != 1 && a.row && 4 * t + hn < heads && f0 == 0) {        // lane (head, quarter, g): four of its sixteen tokens
        float z[4];
        quarter(x[t], pc, z);
        half_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = f32_to_half_sat(z[e]);
        const int tok = 16 * g + 4 * pc;
        half_t* rp = a.row + ((size_t)b * a.H + head0 + 4 * t + hn) * a.Lk + col * PG_TOK + tok;
        if (tok + 4 <= n_here) {
          typedef _Float16 f16x4_ __attribute__((ext_vector_type(4)));
          *(c8_u64_a2*)rp = __builtin_bit_cast(unsigned long long, f16x4_{y[0], y[1], y[2], y[3]});
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (tok + e < n_here) rp[e] = y[e];
        }
      }
      if (n_here < PG_TOK) {                                 // (wave-uniform)
#pragma unroll
        for (int f = 0; f < 16; ++f) x[t][f] = 16 * g + f < n_here ? x[t][f] : -INFINITY;
      }
      float mx = x[t][0];
#pragma unroll
      for (int f = 1; f < 16; ++f) mx = fmaxf(mx, x[t][f]);
      mx = groups_reduce(mx, [](float p, float q) { return fmaxf(p, q); });
      const float m_new = fmaxf(m_run[t], mx);
      // (the maximum is subtracted before the change of base; no key may have been seen yet)
      const float m0 = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = fast_exp2((m_run[t] - m0) * LOG2E);
      m_run[t] = m_new;
      float p[16], ps = 0.f;
#pragma unroll
      for (int f = 0; f < 16; ++f) {
        p[f] = fast_exp2((x[t][f] - m0) * LOG2E);
        ps += p[f];
      }
      l_run[t] = l_run[t] * alpha + ps;
      prob_pieces<FMT>(p, pc, pop[t]);
      if (__any(alpha != 1.f)) {                             // the running maximum rarely moves
        float al[4] = {dpp_move<0x00>(alpha), dpp_move<0x55>(alpha), dpp_move<0xAA>(alpha), dpp_move<0xFF>(alpha)};
#pragma unroll
        for (int d = 0; d < NT; ++d)
#pragma unroll
          for (int v = 0; v < GH; ++v) o[t][d][v] *= al[v];
      }
    }
    if (FMT == 1 && n_here < PG_TOK) {                       // what lies behind the end may be any code, NaN among them
      const int nv = n_here - 16 * g;                          // tokens of this lane's sixteen
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int k = min(max(nv - 4 * q, 0), 4);
        const unsigned keep = k == 4 ? ~0u : (1u << (8 * k)) - 1u;
#pragma unroll
        for (int d = 0; d < NT; ++d) vreg[d][q] &= keep;
      }
    }
    const float w = pw * v_scale;
#pragma unroll
    for (int t = 0; t < GT; ++t)
#pragma unroll
      for (int d = 0; d < NT; ++d) {
        typename M::acc r = M::mul(pop[t][0], vreg[d][0] | (unsigned long long)vreg[d][1] << 32, M::zero());
        r = M::mul(pop[t][1], vreg[d][2] | (unsigned long long)vreg[d][3] << 32, r);
#pragma unroll
        for (int v = 0; v < GH; ++v) o[t][d][v] += (float)r[v] * w;
      }
    if constexpr (MORE) load_v(next);
  };
  if (todo) {
    todo &= todo - 1;
    while (todo) {
      const int next = __builtin_ctzll(todo);
      todo &= todo - 1;
      step(i, next, std::true_type{});
      i = next;
    }
    step(i, 0, std::false_type{});
  }
  // ---- the waves' results
  auto sum = [](float p, float q) { return p + q; };
#pragma unroll
  for (int t = 0; t < GT; ++t) {
    const float l = groups_reduce(l_run[t], sum);
    if (lane < 4) ml_s[wv][4 * t + lane][0] = m_run[t], ml_s[wv][4 * t + lane][1] = l;
#pragma unroll
    for (int d = 0; d < NT; ++d)
#pragma unroll
      for (int v = 0; v < GH; ++v) {
        const float y = groups_reduce(o[t][d][v], sum);      // over the pieces
        if (g == (d & 3)) o_s[wv][t * GH + v][16 * d + n] = y;
      }
  }
  __syncthreads();
  for (int e = tid; e < GT * GH * DK; e += 64 * NW) {
    const int hs = e / DK, f = e % DK, hl = hs / GH * 4 + hs % GH;   // head of the workgroup
    if (hl >= heads) continue;
    float mm = -INFINITY, den = 0.f, num = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) mm = fmaxf(mm, ml_s[w][hl][0]);
    const float m0 = mm == -INFINITY ? 0.f : mm;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float k = fast_exp2((ml_s[w][hl][0] - m0) * LOG2E);   // (a wave without keys: 0)
      den += k * ml_s[w][hl][1];
      num += k * o_s[w][hs][f];
    }
    const int h = head0 + hl;
    if (a.n_span > 1) {
      const size_t at = ((size_t)b * a.n_span + span) * a.H + h;
      a.part_o[at * dk + f0 + f] = num;
      if (f0 + f == 0) a.part_ml[at * 2] = m0, a.part_ml[at * 2 + 1] = den;
    } else {
      const float y = den == 0.f ? 0.f : num / den;
      const size_t at = ((size_t)b * a.H + h) * dk + f0 + f;
      if (a.out_f32) ((float*)a.out)[at] = y;
      else elem<bf16_t>::store((bf16_t*)a.out + at, y);
    }
  }
}

// out = the spans of a sequence merged.  grid (H, B), block DK.  A lane has a span's maximum and sum, 64 at a time; loads of eight spans in flight.
template <int DK>
__global__ __launch_bounds__(DK) void k_cache8_combine(const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                       const int* __restrict__ lens, void* __restrict__ out, int H, int Lk, int n_span,
                                                       int span_tokens, int out_f32) {
  constexpr float LOG2E = 1.4426950408889634f;
  const int h = blockIdx.x, b = blockIdx.y, f = threadIdx.x, lane = f & 63;
  const int len = max(min(lens[b], Lk), 0), n = (len + span_tokens - 1) / span_tokens;
  const size_t at = (size_t)b * n_span * H + h;
  float mm = -INFINITY, num = 0.f, den = 0.f;
  for (int s0 = 0; s0 < n; s0 += 64) {
    const int mine = min(s0 + lane, n - 1);
    const float2 ml = *(const float2*)(part_ml + (at + (size_t)mine * H) * 2);
    const bool in = s0 + lane < n && ml.y != 0.f;
    float m = in ? ml.x : -INFINITY;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    m = fmaxf(m, mm);
    if (m == -INFINITY) continue;                            // (no key yet)
    const float alpha = fast_exp2((mm - m) * LOG2E), k = in ? fast_exp2((ml.x - m) * LOG2E) : 0.f;
    float l = in ? k * ml.y : 0.f;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o, 64);
    mm = m;
    den = den * alpha + l;
    num *= alpha;
    const int cnt = min(64, n - s0);
    for (int s = 0; s < cnt; s += 8) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = part_o[(at + (size_t)(s0 + min(s + u, cnt - 1)) * H) * DK + f];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k), min(s + u, 63)));
        if (s + u < cnt) num += w * x[u];
      }
    }
  }
  const float y = den == 0.f ? 0.f : num / den;
  if (out_f32) ((float*)out)[((size_t)b * H + h) * DK + f] = y;
  else elem<bf16_t>::store((bf16_t*)out + ((size_t)b * H + h) * DK + f, y);
}

}  // namespace lisa
