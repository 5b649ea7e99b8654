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
// (W / 4 lanes, at most 64, per row).  src(h): the row, null: zeros.
template <int FMT, int W, class Src>
__device__ __forceinline__ void stage_queries(int H, int n, unsigned char* codes, int* exps, int tid, int nthreads, Src&& src) {
  constexpr int LPR = W / 4;                                 // lanes per row (a power of two)
  static_assert(LPR <= 64 && (LPR & (LPR - 1)) == 0, "lanes per row");
  for (int e0 = 0; e0 < H * LPR; e0 += nthreads) {           // (nthreads is a multiple of LPR: whole rows)
    const int h = (e0 + tid) / LPR, l = tid % LPR;
    const bf16_t* q = h < H ? src(h) : nullptr;
    float x[4], m = 0.f;
    int bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = q && 4 * l + i < n ? elem<bf16_t>::load(q + 4 * l + i) : 0.f;
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
}

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
      w[q] = pc == 0 ? c[0] : pc == 1 ? c[1] : pc == 2 ? c[2] : 0u;
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
  const bf16_t* w1;           // [Din,F], [F,H]; or
  const bf16_t* w2;
  const unsigned short* img;  // the same in operand order (ffn_operand_piece<false>), if not null
  half_t* row;                // [B,H,Lk] or null
  float* s;                   // [B,H,Lp]
  int H, Lk, Lp, F, fmt;
  float scale;
};
constexpr int C8_SROW = PG_TOK + 4;                          // floats per head of the a_delta tile
constexpr int cache8_scores_lds(int H, int ks, int w_bytes) {
  return (H * C8_SROW + (H + 3) / 4 * 4) * 4 + H * 3 * 32 * ks + w_bytes;
}

// MODE 0: A_n = A_{n-1} + A_delta, 1: FFN(A_{n-1}) + A_delta, 2: FFN([A_{n-1}; A_delta]).  KS: pieces of 32 features of a K_LR row.
// grid (ceil(Lk / 64), B), block 256: a page of a sequence, all heads.  The waves take tiles of four heads in turn (A_delta to the LDS), then
// 16 tokens each through the FFN.  float32 A_n to `s` for k_cache8_pv.
// KVT: key/value heads that the four heads of a tile can have, 1 (groups of whole tiles) or 4; their products go into one accumulator, so that what
// follows on the vector ALU (16 sums over the pieces) is done once per tile.
template <int HBI, int FS, int HBO, int ACT, int MODE, int KS, int KVT>
__global__ __launch_bounds__(256) void k_cache8_scores_mfma(Cache8ScoresArgs a) {
  typedef MfmaFfn<HBI, FS, HBO, ACT> Ffn;
  constexpr int KX = MODE == 0 ? 1 : Ffn::KS;
  extern __shared__ __align__(16) float c8_lds[];
  const Cache8View& c = a.c;
  const int H = a.H, Din = MODE == 2 ? 2 * H : H;
  float* a_s = c8_lds;                                       // [H][C8_SROW]
  int* e_s = (int*)(a_s + H * C8_SROW);                      // [H]
  unsigned char* q_s = (unsigned char*)(e_s + (H + 3) / 4 * 4);   // [H][3][32 KS]
  unsigned short* w_s = (unsigned short*)(q_s + H * 3 * 32 * KS);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = blockIdx.x, b = blockIdx.y;
  const int len = min(c.lens[b], a.Lk);
  if (col * PG_TOK >= len) return;
  const int page = c.page_of(b, col);
  if (page < 0) return;
  const int n = lane & 15, g = lane >> 4;
  const int pj = 16 * wv + n, j = col * PG_TOK + pj;         // this lane's token in the FFN
  const int group = H / c.Hkv, tiles = (H + 3) / 4;
  const int hn = n & 3, pc = n >> 2;
  // keys: the tiles of this wave, UN of them in flight
  constexpr int UN = KVT == 1 ? 4 : KS == 1 ? 2 : 1;
  const int np = c.w8 / 8;
  struct Tile {
    c8_u32x4 k[KVT][KS][2];
    float scale;                                             // of this lane's head
  };
  Tile in[UN];
  auto load_k = [&](int tile, Tile& t) {
    const int first = min(4 * tile, H - 1), kv0 = first / group, kv1 = min(4 * tile + 3, H - 1) / group;
    t.scale = c.k_scale[(size_t)page * c.Hkv + min(4 * tile + hn, H - 1) / group];
#pragma unroll
    for (int v = 0; v < KVT; ++v) {
      const unsigned char* kb = c.k_block(page, min(kv0 + v, kv1));
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u) t.k[v][s][u] = c8_stream(kb + (min(4 * s + g, np - 1) * PG_TOK + page_token(n, u)) * 8);
    }
  };
#pragma unroll
  for (int i = 0; i < UN; ++i) load_k(wv + 4 * i, in[i]);
  // A_{n-1} of this lane's token: what the FFN takes (clamped; past the heads and the end it is zeroed below)
  f16x8 x[1][KX];
  if (MODE != 0)
#pragma unroll
    for (int ks = 0; ks < KX; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[0][ks][e] = a.prev[((size_t)b * H + min(32 * ks + 8 * g + e, H - 1)) * a.Lk + min(j, len - 1)];
  auto src = [&](int h) { return a.q + ((size_t)b * H + h) * c.w; };
  if (a.fmt) stage_queries<1, 32 * KS>(H, c.w, q_s, e_s, tid, 256, src);
  else stage_queries<0, 32 * KS>(H, c.w, q_s, e_s, tid, 256, src);
  if (MODE != 0) {
    if (a.img) Ffn::stage(a.img, w_s, tid, 256);
    else Ffn::stage(a.w1, a.w2, Din, a.F, w_s, tid, 256, 0, H, H);
  }
  __syncthreads();
  auto delta = [&](auto fmt, int tile, const Tile& t) __attribute__((always_inline)) {
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
    if (4 * tile + hn < H) {                                 // lane (head, quarter, g): four of its sixteen tokens
      f32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = pc == 0 ? xs[i] : pc == 1 ? xs[4 + i] : pc == 2 ? xs[8 + i] : xs[12 + i];
      *(f32x4*)(a_s + h * C8_SROW + 16 * g + 4 * pc) = y;
    }
  };
  for (int t0 = wv; t0 < tiles; t0 += 4 * UN) {
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int tile = t0 + 4 * i;
      if (tile < tiles) {
        if (a.fmt) delta(std::integral_constant<int, 1>{}, tile, in[i]);
        else delta(std::integral_constant<int, 0>{}, tile, in[i]);
      }
      if (t0 + 4 * UN < tiles) load_k(tile + 4 * UN, in[i]);
    }
  }
  __syncthreads();
  if constexpr (MODE == 0) {
    for (int e = tid; e < H * PG_TOK; e += 256) {
      const int h = e >> 6, t = e & 63, jt = col * PG_TOK + t;
      if (jt >= len) continue;
      const size_t at = ((size_t)b * H + h) * a.Lk + jt;
      const float y = (float)a.prev[at] + a_s[h * C8_SROW + t];
      if (a.row) a.row[at] = f32_to_half_sat(y);
      a.s[((size_t)b * H + h) * a.Lp + jt] = y;
    }
  } else {
#pragma unroll
    for (int ks = 0; ks < KX; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int ch = 32 * ks + 8 * g + e;
        if (MODE == 2 && ch >= H) x[0][ks][e] = ch < Din ? f32_to_half_sat(a_s[(ch - H) * C8_SROW + pj]) : (_Float16)0.f;
        else if (ch >= Din) x[0][ks][e] = (_Float16)0.f;
      }
    f32x4 y[1][HBO];
    if (MODE == 2) Ffn::template apply_lds_lean<1>(w_s, x, y);
    else Ffn::template apply_lds<1>(w_s, x, y);
    if (j >= len) return;
    float* sp = a.s + (size_t)b * H * a.Lp + j;
    half_t* rp = a.row + (size_t)b * H * a.Lk + j;
#pragma unroll
    for (int hb = 0; hb < HBO; ++hb)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int h = 16 * hb + 4 * g + v;
        if (h >= H) continue;
        const float an = y[0][hb][v] + (MODE == 2 ? 0.f : a_s[h * C8_SROW + pj]);
        sp[(size_t)h * a.Lp] = an;
        if (a.row) rp[(size_t)h * a.Lk] = f32_to_half_sat(an);
      }
  }
}

// ---- softmax and P V --------------------------------------------------------------------------------
struct Cache8PvArgs {
  Cache8View c;
  const bf16_t* q;        // MODE 0: [B,H,DK]
  const float* s;         // MODE 1: A_n [B,H,Lp]
  const half_t* prev;     // MODE 2: A_n [B,H,Lk]
  half_t* row;            // MODE 0, 2: A_n out [B,H,Lk] or null
  void* out;              // [B,H,DK]
  float* part_o;          // [B][n_span][H][DK]   (n_span > 1)
  float* part_ml;         // [B][n_span][H][2]
  int H, Lk, Lp, n_span, span_pages, out_f32;
  int chunks;             // workgroups that the query heads of a key/value head are dealt to, 4 GT each
  float scale;
};

// MODE 0: a standard layer (scores from K), 1: scores given in float32, 2: in half, emitted as they are.
// grid (Hkv chunks, n_span, B), block 64 NW: the pages of a span are dealt to the waves, each with softmax state and sums of its own,
// merged through the LDS at the end; spans by k_cache8_combine.  Bound: the stream of K and V (a page of a head is loaded where the
// one before it has been used, so that every wave has loads in flight); the vector ALU needs 100 - 200 instructions for the
// 8 or 16 KB of a step.
// GT: tiles of four query heads, GH: heads of a tile that are there (1: one query head per key/value head).
template <int FMT, int DK, int MODE, int GT, int GH, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 && GT == 1 && GH == 1 && MODE < 2 ? (MODE == 1 ? 4 : 3) : 1) void k_cache8_pv(Cache8PvArgs a) {
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
  const int b = blockIdx.z, span = blockIdx.y, kv = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int group = a.H / c.Hkv, h0 = chunk * 4 * GT, heads = min(4 * GT, group - h0);   // heads of this workgroup
  const int head0 = kv * group + h0;
  const int len = max(min(c.lens[b], a.Lk), 0), n_pages = (len + PG_TOK - 1) / PG_TOK;
  const int p_begin = span * a.span_pages, p_end = min(n_pages, p_begin + a.span_pages);
  if (p_begin >= n_pages && a.n_span > 1) return;            // (k_cache8_combine knows)
  // lane i: page p_begin + wv + NW i (span_pages <= 64 NW)
  const int my_col = p_begin + wv + NW * lane;
  const int id = my_col < p_end ? c.page_of(b, my_col) : -1;
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
    const unsigned char* vb = c.v_block(__builtin_amdgcn_readlane(id, i), kv) + n * PG_TOK + 16 * g;
#pragma unroll
    for (int t = 0; t < NT; ++t) vreg[t] = c8_stream(vb + t * (16 * PG_TOK));
  };
  auto load_s = [&](int i) {
    const int j = (p_begin + wv + NW * i) * PG_TOK + 16 * g;
    if constexpr (MODE == 1) {
#pragma unroll
      for (int t = 0; t < GT; ++t) {
        const float* sp = a.s + ((size_t)b * a.H + head0 + min(4 * t + hn, heads - 1)) * a.Lp + j;
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
  int i = todo ? __builtin_ctzll(todo) : 0;
  if (todo) {
    load_k(i);
    load_s(i);
    load_v(i);
  }
  unsigned long long qc[MODE == 0 ? GT : 1][KS];
  float qw[MODE == 0 ? GT : 1];
  if constexpr (MODE == 0) {
    stage_queries<FMT, DK>(GT * 4, DK, q_s, e_s, tid, 64 * NW,
                           [&](int h) { return h < heads ? a.q + ((size_t)b * a.H + head0 + h) * DK : nullptr; });
    __syncthreads();
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
      if (MODE != 1 && a.row && 4 * t + hn < heads) {        // lane (head, quarter, g): four of its sixteen tokens
        half_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          y[e] = f32_to_half_sat(pc == 0 ? x[t][e] : pc == 1 ? x[t][4 + e] : pc == 2 ? x[t][8 + e] : x[t][12 + e]);
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
      a.part_o[at * DK + f] = num;
      if (f == 0) a.part_ml[at * 2] = m0, a.part_ml[at * 2 + 1] = den;
    } else {
      const float y = den == 0.f ? 0.f : num / den;
      const size_t at = ((size_t)b * a.H + h) * DK + f;
      if (a.out_f32) ((float*)a.out)[at] = y;
      else elem<bf16_t>::store((bf16_t*)a.out + at, y);
    }
  }
}

// out = the spans of a sequence merged.  grid (H, B), block DK.
template <int DK>
__global__ __launch_bounds__(DK) void k_cache8_combine(const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                       const int* __restrict__ lens, void* __restrict__ out, int H, int Lk, int n_span,
                                                       int span_tokens, int out_f32) {
  constexpr float LOG2E = 1.4426950408889634f;
  const int h = blockIdx.x, b = blockIdx.y, f = threadIdx.x;
  const int len = max(min(lens[b], Lk), 0), n = (len + span_tokens - 1) / span_tokens;
  const size_t at = (size_t)b * n_span * H + h;
  float mm = -INFINITY;
  for (int s = 0; s < n; ++s) {
    const float2 ml = *(const float2*)(part_ml + (at + (size_t)s * H) * 2);
    if (ml.y != 0.f) mm = fmaxf(mm, ml.x);
  }
  float num = 0.f, den = 0.f;
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const float2 ml = *(const float2*)(part_ml + (at + (size_t)s * H) * 2);
    const float k = ml.y != 0.f ? fast_exp2((ml.x - mm) * LOG2E) : 0.f;
    num += k * part_o[(at + (size_t)s * H) * DK + f];
    den += k * ml.y;
  }
  const float y = den == 0.f ? 0.f : num / den;
  if (out_f32) ((float*)out)[((size_t)b * H + h) * DK + f] = y;
  else elem<bf16_t>::store((bf16_t*)out + ((size_t)b * H + h) * DK + f, y);
}

}  // namespace lisa
