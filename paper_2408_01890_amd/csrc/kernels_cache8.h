// The paged 8-bit cache (Sec. 5.2: what the decoding stage keeps of K_LR, or K, and V): appending tokens to it, and the
// shape-generic kernels of a decode step over it.
//
// A page holds 64 tokens of a layer. Per page and key/value head:
//   K  [ceil(w / 8)][64][8]  codes of the key rows, features in pieces of 8 (the last one filled up with zeros): 8 bytes of a
//                            token are what a lane of the 16x16x32 8-bit MFMAs holds of an operand row
//   V  [d_k][64]             codes of the value rows, tokens innermost: the keys are what P V sums over
//   one scale each, a power of two: code c stands for c * scale.
// The scale of a block is 2^e with the smallest e >= -126 for which the block's largest finite |x| is at most top * 2^e (top =
// 127: whole numbers, 448: e4m3).  When a token arrives that does not fit, the scale grows and the block's codes are rounded
// again.  Powers of two keep that harmless: a code loses bits by halves, so the error stays within one step of the
// final scale however often it grows, and every product with a scale is exact.  (With s = max / 127 a code of 10 is
// rounded back to 10 at each growth by 4 %, and stands for twice the value after 18 of them.)
#pragma once
#include "kernels_generic.h"

namespace lisa {

constexpr int PG_TOK = 64;       // LISA_PAGE_TOKENS

// ---- codes ------------------------------------------------------------------------------------
// FMT: lisa_cache_format.
template <int FMT> struct code8;
template <> struct code8<0> {                                // whole numbers
  static constexpr unsigned TOP_MANTISSA = 0x7e0000u;        // 127 = 1.984375 * 2^6
  static constexpr int TOP_EXP = 6;
  static __device__ __forceinline__ float load(unsigned char c) { return (float)(signed char)c; }
  static __device__ __forceinline__ unsigned char store(float x) {   // NaN has no code: 0
    const float y = rintf(__builtin_amdgcn_fmed3f(x, -127.f, 127.f));
    return (unsigned char)(x == x ? (int)y : 0);
  }
  // four numbers within the top
  static __device__ __forceinline__ unsigned store4(float a, float b, float c, float d, float inv) {
    const float M = 12582912.f;                              // 1.5 * 2^23: the sum's low byte is the number rounded
    const unsigned x = __float_as_uint(__builtin_fmaf(a, inv, M)), y = __float_as_uint(__builtin_fmaf(b, inv, M));
    const unsigned z = __float_as_uint(__builtin_fmaf(c, inv, M)), w = __float_as_uint(__builtin_fmaf(d, inv, M));
    return __builtin_amdgcn_perm(y, x, 0x0c0c0400u) | __builtin_amdgcn_perm(w, z, 0x04000c0cu);
  }
};
template <> struct code8<1> {                                // e4m3
  static constexpr unsigned TOP_MANTISSA = 0x600000u;        // 448 = 1.75 * 2^8
  static constexpr int TOP_EXP = 8;
  static __device__ __forceinline__ float load(unsigned char c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }
  static __device__ __forceinline__ unsigned char store(float x) {
    const float y = __builtin_amdgcn_fmed3f(x, -448.f, 448.f);
    return x == x ? (unsigned char)(__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xff) : (unsigned char)0x7f;
  }
  static __device__ __forceinline__ unsigned store4(float a, float b, float c, float d, float inv) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, lo, true);
  }
};

// The scale of a block whose largest finite magnitude is m.
template <int FMT>
__device__ __forceinline__ float block_scale(float m) {
  const unsigned u = __float_as_uint(m);
  int e = (int)(u >> 23) - 127 - code8<FMT>::TOP_EXP + ((u & 0x7fffffu) > code8<FMT>::TOP_MANTISSA ? 1 : 0);
  e = max(e, -126);                                          // (0 and subnormal numbers among them)
  return __uint_as_float((unsigned)(e + 127) << 23);
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

struct Cache8View {
  unsigned char* k;
  float* k_scale;
  unsigned char* v;
  float* v_scale;
  const int* table;      // [B][max_pages]
  const int* lens;       // [B]
  int n_pages, max_pages, Hkv, w, w8, dk;   // w8: w rounded up to 8
  __device__ __forceinline__ unsigned char* k_block(int page, int kv) const { return k + ((size_t)page * Hkv + kv) * (w8 * PG_TOK); }
  __device__ __forceinline__ unsigned char* v_block(int page, int kv) const { return v + ((size_t)page * Hkv + kv) * (dk * PG_TOK); }
  // The page of column `col` of sequence b; negative where there is none.  (The load does not wait for anything.)
  __device__ __forceinline__ int entry(int b, int col) const {
    const int p = table[(size_t)b * max_pages + min(col, max_pages - 1)];
    return col < max_pages && (unsigned)p < (unsigned)n_pages ? p : -1;
  }
};

// ---- append -----------------------------------------------------------------------------------
// Eight features f0 .. f0 + 7 of a row of `width` elements as they lie in memory.  Rows of whole octets are 16-byte aligned.  The loads are apart
// from what is made of them, and clamped to the row, not branched around: all of a thread's are in flight together (with
// each octet turned into numbers where it was loaded, 6 prompts of 1500 tokens took 51 us).
template <typename T>
struct Octet {
  unsigned r[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* row, int f0, int width) {
    typedef unsigned int u32x4_ __attribute__((ext_vector_type(4)));
    if (width % 8 == 0) {
#pragma unroll
      for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        const u32x4_ v = *(const u32x4_*)(row + f0 + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[4 * h + i] = v[i];
      }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = *(const unsigned*)(row + min(f0 + i, width - 1));
    } else if (width % 2 == 0) {                             // (rows are 4-byte aligned)
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = *(const unsigned*)(row + min(f0 + 2 * i, width - 2));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        r[i] = row[min(f0 + 2 * i, width - 1)].bits | (unsigned)row[min(f0 + 2 * i + 1, width - 1)].bits << 16;
    }
  }
  // zeros past the width, and everywhere where the row is not one of the call's
  __device__ __forceinline__ void get(int f0, int width, bool live, float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned u;
      if constexpr (sizeof(T) == 4) u = r[i];
      else u = i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16;
      x[i] = live && f0 + i < width ? __uint_as_float(u) : 0.f;
    }
  }
};
// The largest magnitude as bits (infinities and NaN are the largest ones).
__device__ __forceinline__ unsigned octet_max(const float (&x)[8], unsigned m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ float octet_finite_max(const float (&x)[8], float m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(x[i]));
  return m;
}
// `whole`: no infinity or NaN is among the numbers (and the scale takes them all).
template <int FMT>
__device__ __forceinline__ unsigned quad_codes(float a, float b, float c, float d, float inv, bool whole) {
  typedef code8<FMT> C;
  if (whole) return C::store4(a, b, c, d, inv);
  return C::store(a * inv) | (unsigned)C::store(b * inv) << 8 | (unsigned)C::store(c * inv) << 16 | (unsigned)C::store(d * inv) << 24;
}
template <int FMT>
__device__ __forceinline__ unsigned long long octet_codes(const float (&x)[8], float inv, bool whole) {
  return quad_codes<FMT>(x[0], x[1], x[2], x[3], inv, whole) |
         (unsigned long long)quad_codes<FMT>(x[4], x[5], x[6], x[7], inv, whole) << 32;
}
__device__ __forceinline__ unsigned wave_max_bits(unsigned v) {
  return __float_as_uint(wave_reduce(__uint_as_float(v), [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }));
}

// The last counts[b] tokens of sequence b (all L rows where counts is null) go into its pages.
// grid (pages that L tokens can touch, Hkv, B), block 256: a workgroup has one page of one head.  Its new rows are read once, into
// registers (a thread: eight features of four tokens), for the largest magnitudes and then the codes; values are turned
// through the LDS into rows of tokens.  WIDE: rows of more than 128 features.  Bound: the stream (6 prompts of up to 1500 tokens, 32 heads,
// 187 MB: 42 us, 4.4 of the 4.8 TB/s of a large copy).
constexpr int C8_VROW = PG_TOK + 4;      // bytes of a feature's row of codes in the LDS
constexpr int C8_KROW = PG_TOK * 8 + 16;  // of an octet's
template <typename T, int FMT, bool WIDE>
__global__ __launch_bounds__(256) void k_cache8_append(Cache8View c, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                       const int* __restrict__ counts, int L) {
  constexpr int N = WIDE ? 2 : 1, FEATURES = N * 128;        // (16 token quads x width / 8 tasks for N * 256 threads)
  __shared__ __align__(16) unsigned char v_s[FEATURES * C8_VROW];
  __shared__ __align__(16) unsigned char k_s[(FEATURES / 8) * C8_KROW];
  __shared__ unsigned m_s[2][4];
  __shared__ float f_s[2][4];
  const int kv = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int len = c.lens[b], n_new = min(max(counts ? counts[b] : L, 0), min(L, len));
  if (n_new <= 0) return;
  const int col = (len - n_new) / PG_TOK + (int)blockIdx.x;
  if ((long long)col * PG_TOK >= len) return;
  const int lo = max(len - n_new - col * PG_TOK, 0), hi = min(len - col * PG_TOK, PG_TOK);   // tokens of the page
  // row of token t of the page: base + t (t >= lo)
  const long long base = ((long long)b * c.Hkv + kv) * L + (col * PG_TOK - (len - n_new));
  const int nv = (c.dk + 7) / 8, nk = c.w8 / 8;
  const bool k_quads = c.w % 8 == 0;                         // else a thread has a token, three octets at most of a K_LR row keep all busy
  // The rows (they are on their way while the table is asked for the page).
  auto row_of = [&](int t) { return base + min(max(t, lo), hi - 1); };
  auto live = [&](int t) { return t >= lo && t < hi; };
  const int t_k = tid & 63;
  Octet<T> rv[N][4], rk[N][4];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = tid + 256 * i, q = e / nv, o = e % nv;     // token quad, octet (octets fastest: rows are read on end)
#pragma unroll
    for (int u = 0; u < 4; ++u) rv[i][u].load(v_new + row_of(4 * q + u) * c.dk, 8 * o, c.dk);
  }
  if (k_quads && nk) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = tid + 256 * i, q = e / nk, o = e % nk;
#pragma unroll
      for (int u = 0; u < 4; ++u) rk[i][u].load(k_new + row_of(4 * q + u) * c.w, 8 * o, c.w);
    }
  } else if (nk) {                                           // octets tid / 64 (+ 4, ..: four of them in registers)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (4 * u < nk) rk[0][u].load(k_new + row_of(t_k) * c.w, 8 * min((tid >> 6) + 4 * u, nk - 1), c.w);
  }
  const int page = c.entry(b, col);
  if (page < 0) return;
  const size_t at = (size_t)page * c.Hkv + kv;
  const float k_old = c.w ? c.k_scale[at] : 0.f, v_old = c.v_scale[at];
  float xv[N][4][8], xk[N][4][8];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = tid + 256 * i;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      rv[i][u].get(8 * (e % nv), c.dk, live(4 * (e / nv) + u), xv[i][u]);
      if (k_quads) rk[i][u].get(nk ? 8 * (e % nk) : 0, c.w, nk && live(4 * (e / nk) + u), xk[i][u]);
      else rk[0][u].get(8 * ((tid >> 6) + 4 * u), c.w, 4 * u < nk && live(t_k), xk[0][u]);
    }
  }
  unsigned mk = 0, mv = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      mv = octet_max(xv[i][u], mv);
      if (i == 0 || k_quads) mk = octet_max(xk[i][u], mk);
    }
  if (!k_quads)                                              // (rows of more than 128 features)
    for (int o = (tid >> 6) + 16; o < nk; o += 4)
      if (live(t_k)) {
        float x[8];
        Octet<T> r;
        r.load(k_new + row_of(t_k) * c.w, 8 * o, c.w);
        r.get(8 * o, c.w, true, x);
        mk = octet_max(x, mk);
      }
  mk = wave_max_bits(mk), mv = wave_max_bits(mv);
  if ((tid & 63) == 0) m_s[0][tid >> 6] = mk, m_s[1][tid >> 6] = mv;
  __syncthreads();
  mk = max(max(m_s[0][0], m_s[0][1]), max(m_s[0][2], m_s[0][3]));
  mv = max(max(m_s[1][0], m_s[1][1]), max(m_s[1][2], m_s[1][3]));
  const bool k_whole = mk < 0x7f800000u, v_whole = mv < 0x7f800000u;
  float fk = __uint_as_float(mk), fv = __uint_as_float(mv);
  if (!(k_whole && v_whole)) {                               // the largest finite magnitudes
    fk = 0.f, fv = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        fv = octet_finite_max(xv[i][u], fv);
        if (i == 0 || k_quads) fk = octet_finite_max(xk[i][u], fk);
      }
    if (!k_quads)
      for (int o = (tid >> 6) + 16; o < nk; o += 4)
        if (live(t_k)) {
          float x[8];
          Octet<T> r;
          r.load(k_new + row_of(t_k) * c.w, 8 * o, c.w);
          r.get(8 * o, c.w, true, x);
          fk = octet_finite_max(x, fk);
        }
    fk = wave_max(fk), fv = wave_max(fv);
    if ((tid & 63) == 0) f_s[0][tid >> 6] = fk, f_s[1][tid >> 6] = fv;
    __syncthreads();
    fk = fmaxf(fmaxf(f_s[0][0], f_s[0][1]), fmaxf(f_s[0][2], f_s[0][3]));
    fv = fmaxf(fmaxf(f_s[1][0], f_s[1][1]), fmaxf(f_s[1][2], f_s[1][3]));
  }
  float k_now = block_scale<FMT>(fk), v_now = block_scale<FMT>(fv);
  if (lo) k_now = fmaxf(k_now, k_old), v_now = fmaxf(v_now, v_old);   // (tokens that are there already count too)
  if (tid == 0) {
    if (c.w) c.k_scale[at] = k_now;
    c.v_scale[at] = v_now;
  }
  typedef code8<FMT> Code;
  // values: through the LDS, [feature][token]
  const float v_inv = 1.f / v_now, k_inv = 1.f / k_now;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = tid + 256 * i, q = e / nv, o = e % nv;
    if (q >= 16 || 4 * q >= hi || 4 * q + 4 <= lo) continue;
#pragma unroll
    for (int f = 0; f < 8; ++f)
      if (8 * o + f < c.dk)
        *(unsigned*)(v_s + (8 * o + f) * C8_VROW + 4 * q) = quad_codes<FMT>(xv[i][0][f], xv[i][1][f], xv[i][2][f], xv[i][3][f], v_inv, v_whole);
  }
  // keys: 8 features of a token at a time
  unsigned char* kb = c.k_block(page, kv);
  if (k_quads) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = tid + 256 * i, q = nk ? e / nk : 16, o = nk ? e % nk : 0;
      if (q >= 16) continue;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int t = 4 * q + u;
        if (t >= lo && t < hi) *(unsigned long long*)(k_s + o * C8_KROW + t * 8) = octet_codes<FMT>(xk[i][u], k_inv, k_whole);
      }
    }
  } else if (live(t_k)) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int o = (tid >> 6) + 4 * u;
      if (o < nk) *(unsigned long long*)(kb + (o * PG_TOK + t_k) * 8) = octet_codes<FMT>(xk[0][u], k_inv, k_whole);
    }
    for (int o = (tid >> 6) + 16; o < nk; o += 4) {
      float x[8];
      Octet<T> r;
      r.load(k_new + row_of(t_k) * c.w, 8 * o, c.w);
      r.get(8 * o, c.w, true, x);
      *(unsigned long long*)(kb + (o * PG_TOK + t_k) * 8) = octet_codes<FMT>(x, k_inv, k_whole);
    }
  }
  if (lo && k_now > k_old)
    for (int e = tid; e < lo * nk; e += 256) {
      unsigned long long* at8 = (unsigned long long*)(kb + ((size_t)(e / lo) * PG_TOK + e % lo) * 8);
      const unsigned long long x = *at8;
      unsigned long long y = 0;
      for (int f = 0; f < 8; ++f)
        y |= (unsigned long long)Code::store(Code::load((unsigned char)(x >> (8 * f))) * k_old * k_inv) << (8 * f);
      *at8 = y;
    }
  __syncthreads();
  if (k_quads)                                               // out as rows of tokens, two at a time
    for (int e = tid; e < nk * 32; e += 256) {
      const int o = e >> 5, t = 2 * (e & 31);
      const unsigned long long* src = (const unsigned long long*)(k_s + o * C8_KROW + t * 8);
      unsigned long long* dst = (unsigned long long*)(kb + (o * PG_TOK + t) * 8);
      if (t >= lo && t + 2 <= hi) {
        *(uint4*)dst = *(const uint4*)src;
      } else {
        if (t >= lo && t < hi) dst[0] = src[0];
        if (t + 1 >= lo && t + 1 < hi) dst[1] = src[1];
      }
    }
  unsigned char* vb = c.v_block(page, kv);
  const int from = lo && v_now > v_old ? 0 : lo;              // tokens to write
  if (from < lo) {
    for (int e = tid; e < lo * c.dk; e += 256) {
      const int f = e / lo, t = e % lo;
      v_s[f * C8_VROW + t] = Code::store(Code::load(vb[f * PG_TOK + t]) * v_old * v_inv);
    }
    __syncthreads();
  }
  for (int e = tid; e < c.dk * 4; e += 256) {                // 16 tokens of a feature at a time
    const int f = e >> 2, t = 16 * (e & 3);
    const unsigned* src = (const unsigned*)(v_s + f * C8_VROW + t);
    unsigned char* dst = vb + f * PG_TOK + t;
    if (t >= from && t + 16 <= hi) {
      *(uint4*)dst = make_uint4(src[0], src[1], src[2], src[3]);
    } else if (t < hi && t + 16 > from) {
      for (int u = max(from - t, 0); u < min(hi - t, 16); ++u) dst[u] = ((const unsigned char*)src)[u];
    }
  }
}

// One new token per sequence (L = 1): a wave has a head of a sequence, so nothing waits for other waves: what it takes is the chain lens ->
// table -> scales -> codes.  grid (ceil(Hkv / 4), B), block 256.  (64 sequences, 32 heads: 17.8 us with k_cache8_append, whose threads all load.)
template <typename T, int FMT>
__global__ __launch_bounds__(256) void k_cache8_append_token(Cache8View c, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                             const int* __restrict__ counts) {
  typedef code8<FMT> Code;
  constexpr int E = 4;                                       // elements of a row per lane (256 features at most)
  const int lane = threadIdx.x & 63, kv = blockIdx.x * 4 + (threadIdx.x >> 6), b = blockIdx.y;
  if (kv >= c.Hkv) return;
  const size_t row = (size_t)b * c.Hkv + kv;
  float xk[E], xv[E], mk = 0.f, mv = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int f = lane + 64 * i;
    xk[i] = f < c.w ? elem<T>::load(k_new + row * c.w + f) : 0.f;
    xv[i] = f < c.dk ? elem<T>::load(v_new + row * c.dk + f) : 0.f;
  }
  const int len = c.lens[b], col = (len - 1) / PG_TOK, t = (len - 1) % PG_TOK;
  if (len <= 0 || (counts && counts[b] <= 0)) return;
  const int page = c.entry(b, col);
  if (page < 0) return;
  const size_t at = (size_t)page * c.Hkv + kv;
  const float k_old = c.w ? c.k_scale[at] : 0.f, v_old = c.v_scale[at];
#pragma unroll
  for (int i = 0; i < E; ++i) mk = fmaxf(mk, finite_abs(xk[i])), mv = fmaxf(mv, finite_abs(xv[i]));
  float k_now = block_scale<FMT>(wave_max(mk)), v_now = block_scale<FMT>(wave_max(mv));
  if (t) k_now = fmaxf(k_now, k_old), v_now = fmaxf(v_now, v_old);
  if (lane == 0) {
    if (c.w) c.k_scale[at] = k_now;
    c.v_scale[at] = v_now;
  }
  const float k_inv = 1.f / k_now, v_inv = 1.f / v_now;
  unsigned char* kb = c.k_block(page, kv);
  unsigned char* vb = c.v_block(page, kv);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int f = lane + 64 * i;
    if (f < c.w8) kb[((f >> 3) * PG_TOK + t) * 8 + (f & 7)] = Code::store(xk[i] * k_inv);   // (past the width: zeros)
    if (f < c.dk) vb[f * PG_TOK + t] = Code::store(xv[i] * v_inv);
  }
  if (t && k_now > k_old)                                    // the tokens in front, rounded again
    for (int e = lane; e < c.w8 * t; e += 64) {
      unsigned char* p = kb + ((e / (8 * t)) * PG_TOK + e / 8 % t) * 8 + (e & 7);
      *p = Code::store(Code::load(*p) * k_old * k_inv);
    }
  if (t && v_now > v_old)
    for (int e = lane; e < c.dk * t; e += 64) {
      unsigned char* p = vb + (e / t) * PG_TOK + e % t;
      *p = Code::store(Code::load(*p) * v_old * v_inv);
    }
}

// ---- decode step, any shape ---------------------------------------------------------------------
// Scores of one page (64 keys) of one sequence, all heads; float32 arithmetic.  The stages of k_lisa_scores; `mix` 4: the
// standard layer's q K^T.  exact [B][H][Lk] float32, -inf at keys that have no page; `scores` may be null.
// grid (ceil(Lk / 64), B), block 256.
template <typename T, typename S, int FMT>
__global__ __launch_bounds__(256) void k_cache8_scores(Cache8View c, const T* __restrict__ q, const S* __restrict__ prev,
                                                       const T* __restrict__ w1, const T* __restrict__ w2, S* __restrict__ scores,
                                                       float* __restrict__ exact, int H, int Lk, int F, int mix, int act, float scale) {
  extern __shared__ float c8_sm[];
  const bool concat = mix == 1, has_ffn = mix <= 1, has_delta = mix != 3, has_prev = mix != 4;
  const int Din = concat ? 2 * H : H;
  float* xs = c8_sm;
  float* hs = xs + Din * 64;
  float* ds = hs + F * 64;
  const int col = blockIdx.x, b = blockIdx.y;
  const int len = min(c.lens[b], Lk);
  const int pj = threadIdx.x & 63, sl = threadIdx.x >> 6;
  const int j = col * PG_TOK + pj;
  if (col * PG_TOK >= len) return;
  const int page = c.entry(b, col);
  const bool live = j < len && page >= 0;
  const int group = H / c.Hkv;
  const size_t row = (size_t)b * H * Lk + j;                 // + h * Lk
  for (int h = sl; h < H; h += 4) {
    float acc = 0.f, x = 0.f;
    if (live) {
      if (has_delta) {
        const T* qp = q + ((size_t)b * H + h) * c.w;
        const unsigned char* kp = c.k_block(page, h / group) + pj * 8;
        for (int t = 0; t < c.w; ++t) acc += elem<T>::load(qp + t) * code8<FMT>::load(kp[(t >> 3) * (PG_TOK * 8) + (t & 7)]);
        acc *= c.k_scale[(size_t)page * c.Hkv + h / group] * scale;
      }
      if (has_prev) x = elem<S>::load(prev + row + (size_t)h * Lk);
    }
    if (!has_ffn) {
      if (live && scores) elem<S>::store(scores + row + (size_t)h * Lk, x + acc);
      if (j < len) exact[row + (size_t)h * Lk] = live ? x + acc : -INFINITY;
      continue;
    }
    ds[h * 64 + pj] = acc;
    xs[h * 64 + pj] = x;
    if (concat) xs[(H + h) * 64 + pj] = acc;
  }
  if (!has_ffn) return;
  __syncthreads();
  for (int f = sl; f < F; f += 4) {
    float acc = 0.f;
    for (int ch = 0; ch < Din; ++ch) acc += xs[ch * 64 + pj] * elem<T>::load(w1 + (size_t)ch * F + f);
    hs[f * 64 + pj] = act == 0 ? fmaxf(acc, 0.f) : act == 1 ? acc / (1.f + expf(-acc)) : acc;
  }
  __syncthreads();
  for (int h = sl; h < H; h += 4) {
    float acc = 0.f;
    if (act == 2) {
      acc = hs[h * 64 + pj];
    } else {
      for (int f = 0; f < F; ++f) acc += hs[f * 64 + pj] * elem<T>::load(w2 + (size_t)f * H + h);
    }
    if (!concat) acc += ds[h * 64 + pj];
    if (live && scores) elem<S>::store(scores + row + (size_t)h * Lk, acc);
    if (j < len) exact[row + (size_t)h * Lk] = live ? acc : -INFINITY;
  }
}

// Softmax over the tokens of a sequence and P V, one head of one sequence per workgroup; float32 arithmetic, zeros where no
// key is seen.  grid (H, B), block 256 (d_k <= 256).
template <typename T, typename O, int FMT>
__global__ __launch_bounds__(256) void k_cache8_softmax_v(Cache8View c, const float* __restrict__ exact, O* __restrict__ out, int H, int Lk) {
  __shared__ float p_s[PG_TOK], alpha_s;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int kv = h / (H / c.Hkv), len = min(c.lens[b], min(Lk, c.max_pages * PG_TOK));
  const float* a = exact + ((size_t)b * H + h) * Lk;
  float m_run = -INFINITY, l_run = 0.f, acc = 0.f;           // (m_run, l_run: the first wave)
  for (int col = 0; col * PG_TOK < len; ++col) {
    const int page = c.entry(b, col);
    if (page < 0) continue;                                  // (uniform)
    if (tid < 64) {
      const int j = col * PG_TOK + tid;
      const float s = j < len ? a[j] : -INFINITY;
      const float m_new = fmaxf(m_run, wave_max(s));
      const float m0 = m_new == -INFINITY ? 0.f : m_new;
      const float p = j < len ? __expf(s - m0) : 0.f;
      const float alpha = __expf(m_run - m0);
      l_run = l_run * alpha + wave_sum(p);
      m_run = m_new;
      p_s[tid] = p;
      if (tid == 0) alpha_s = alpha;
    }
    __syncthreads();
    if (tid < c.dk) {
      const unsigned char* vp = c.v_block(page, kv) + tid * PG_TOK;
      const int n = min(PG_TOK, len - col * PG_TOK);
      float t = 0.f;
      for (int u = 0; u < n; ++u) t += p_s[u] * code8<FMT>::load(vp[u]);
      acc = acc * alpha_s + t * c.v_scale[(size_t)page * c.Hkv + kv];
    }
    __syncthreads();
  }
  if (tid == 0) alpha_s = l_run == 0.f ? 0.f : 1.f / l_run;   // (NaN stays NaN)
  __syncthreads();
  if (tid < c.dk) elem<O>::store(out + ((size_t)b * H + h) * c.dk + tid, acc * alpha_s);
}

}  // namespace lisa
