// Pages of the 8-bit caches: which sequence has which (k_pages_*), and moving what is in them (k_pages_copy).
//
// State: table [S][C], the page of tokens 64 c .. 64 c + 63 of sequence s (-1: none); lens [S]; refs [P], how often a page is
// named (0: free).  One table serves the pools of all layers.  Every choice is a rule on indices (the free page with the lowest
// number first, sequences and requests in their order), so results do not depend on scheduling.  The state is a few
// hundred KB at most, and what a call decides depends on prefix sums over all of it: one workgroup of 1024 threads (64 sequences, 8192 pages: free
// 2.1 us, grow 5).
#pragma once
#include "lisa_types.h"

namespace lisa {

constexpr int PGS_THREADS = 1024;

struct PagesView {
  int* table;
  int* lens;
  int* refs;
  int P, S, C;
  // workspace
  int* owner;      // [S] which request names a sequence first
  int* info;       // [S] lengths before the call
  int* ids;        // [2 P] free pages in ascending order (as many as are wanted); compaction: where pages go, and which
};
__device__ __forceinline__ int pages_of(int tokens) { return (int)(((long long)tokens + 63) / 64); }

// Inclusive prefix sum over the workgroup and its total.
struct PgsScan {
  int wave[PGS_THREADS / 64];
};
__device__ __forceinline__ int pgs_scan(int v, int& total, PgsScan& s) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  __syncthreads();                                           // (the scan before has been read)
  if (lane == 63) s.wave[wv] = v;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < PGS_THREADS / 64; ++w) {
    if (w < wv) before += s.wave[w];
    total += s.wave[w];
  }
  return before + v;
}

// The counts of eight pages per thread, of 8192 in all.  A kernel asks for the first 8192 (`first`) when it begins, beside what else it reads: what it
// spends is a chain of reads and barriers of about a microsecond each.
constexpr int PGS_EACH = 8;
struct PgsRefs {
  int r[PGS_EACH];
  __device__ __forceinline__ void load(const PagesView& g, int p0) {
    typedef int i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
    const int p = p0 + PGS_EACH * (int)threadIdx.x;
    if (p + PGS_EACH <= g.P) {
#pragma unroll
      for (int q = 0; q < PGS_EACH / 4; ++q) {
        const i32x4_a4 x = *(const i32x4_a4*)(g.refs + p + 4 * q);
#pragma unroll
        for (int u = 0; u < 4; ++u) r[4 * q + u] = x[u];
      }
    } else {
#pragma unroll
      for (int u = 0; u < PGS_EACH; ++u) r[u] = g.refs[min(p + u, g.P - 1)];
    }
  }
};
// A list of pages, the first 2048 of them in the LDS.
constexpr int PGS_LDS_IDS = 2048;
struct PgsList {
  int* lds;
  int* rest;               // [P] of the workspace
  __device__ __forceinline__ void put(int i, int p) const {
    if (i < PGS_LDS_IDS) lds[i] = p;
    else rest[i] = p;
  }
  __device__ __forceinline__ int get(int i) const { return i < PGS_LDS_IDS ? lds[i] : rest[i]; }
};
// list[0 .. n) = the first pages in [from, to) for which pick(refs) holds, n <= want of them; returns n.  (Every thread calls it.)
template <class Pick>
__device__ __forceinline__ int pgs_collect(const PagesView& g, const PgsRefs& first, int from, int to, int want, const PgsList& list, PgsScan& s,
                                           Pick&& pick) {
  constexpr int CHUNK = PGS_EACH * PGS_THREADS;
  int found = 0;
  for (int p0 = from / CHUNK * CHUNK; p0 < to && found < want; p0 += CHUNK) {
    PgsRefs x = first;
    if (p0) x.load(g, p0);
    const int p = p0 + PGS_EACH * (int)threadIdx.x;
    unsigned in = 0;
#pragma unroll
    for (int u = 0; u < PGS_EACH; ++u) in |= (p + u >= from && p + u < to && pick(x.r[u]) ? 1u : 0u) << u;
    const int n = __popc(in);
    int total, at = found + pgs_scan(n, total, s) - n;
#pragma unroll
    for (int u = 0; u < PGS_EACH; ++u)
      if (in >> u & 1) {
        if (at < want) list.put(at, p + u);
        ++at;
      }
    found += total;
  }
  __syncthreads();
  return min(found, want);
}

// owner(s) = the first request that names s, in the LDS where 2048 sequences are all.
constexpr int PGS_LDS_OWNERS = 2048;
__device__ __forceinline__ int* pgs_owners_clear(const PagesView& g, int* lds, int n) {
  int* owner = g.S <= PGS_LDS_OWNERS ? lds : g.owner;
  for (int s = threadIdx.x; s < g.S; s += PGS_THREADS) owner[s] = n;
  __syncthreads();
  return owner;
}

// Sequence s is given add[s] more tokens and the pages they need.
__global__ __launch_bounds__(PGS_THREADS) void k_pages_grow(PagesView g, const int* __restrict__ add, int* __restrict__ done) {
  __shared__ PgsScan scan;
  __shared__ int base_s[PGS_THREADS], more_s[PGS_THREADS], have_s[PGS_THREADS], ids_s[PGS_LDS_IDS];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  PgsRefs first;
  first.load(g, 0);
  int len, inc, more;                                        // of sequence s0 + tid: its tokens, those added, the pages they need
  auto read = [&](int s0) {
    const int s = min(s0 + tid, g.S - 1);
    len = g.lens[s], inc = add[s];
    const long long want = (long long)len + inc;
    const bool ok = s0 + tid < g.S && inc >= 0 && len >= 0 && want <= (long long)g.C * 64;
    more = ok ? pages_of((int)want) - pages_of(len) : 0;
    return ok;
  };
  const bool one = g.S <= PGS_THREADS;                       // (all sequences at once: they are read once)
  int want = 0;                                              // pages wanted by all (no more than there are)
  bool ok = false;
  for (int s0 = 0; s0 < g.S; s0 += PGS_THREADS) {
    int total;
    ok = read(s0);
    (void)pgs_scan(min(more, g.P), total, scan);
    want = (int)min((long long)want + total, (long long)g.P);
  }
  const PgsList ids{ids_s, g.ids};
  const int found = pgs_collect(g, first, 0, g.P, want, ids, scan, [](int r) { return r == 0; });
  long long given = 0;
  for (int s0 = 0; s0 < g.S; s0 += PGS_THREADS) {
    const int s = s0 + tid;
    if (!one) ok = read(s0);
    int total;
    const int capped = min(more, g.P + 1);                   // (no sum of 1024 of them passes 32 bits: P is at most 2^20)
    const long long upto = given + pgs_scan(capped, total, scan);
    const bool yes = ok && (more == 0 || upto <= found);
    base_s[tid] = (int)(upto - capped);
    more_s[tid] = yes ? more : 0;
    have_s[tid] = pages_of(max(len, 0));
    given += total;
    __syncthreads();
    for (int u = wv; u < PGS_THREADS && s0 + u < g.S; u += PGS_THREADS / 64) {
      const int m = more_s[u];
      for (int c = lane; c < m; c += 64) {
        const int p = ids.get(base_s[u] + c);
        g.table[(size_t)(s0 + u) * g.C + have_s[u] + c] = p;
        g.refs[p] = 1;
      }
    }
    __syncthreads();                                         // (the next 1024 use the same LDS)
    if (s < g.S) {
      if (yes) g.lens[s] = len + inc;
      done[s] = yes;
    }
  }
}

// The sequences named give their pages back.
__global__ __launch_bounds__(PGS_THREADS) void k_pages_free(PagesView g, const int* __restrict__ seqs, int n, int* __restrict__ done) {
  __shared__ int owner_s[PGS_LDS_OWNERS];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  int* owner = pgs_owners_clear(g, owner_s, n);
  for (int i = threadIdx.x; i < n; i += PGS_THREADS)
    if ((unsigned)seqs[i] < (unsigned)g.S) atomicMin(owner + seqs[i], i);
  __syncthreads();
  for (int i = wv; i < n; i += PGS_THREADS / 64) {
    const int s = seqs[i];
    const bool yes = (unsigned)s < (unsigned)g.S && owner[s] == i;
    if (yes) {
      const int have = min(pages_of(max(g.lens[s], 0)), g.C);
      for (int c = lane; c < g.C; c += 64) {
        const int p = g.table[(size_t)s * g.C + c];
        if (c < have && (unsigned)p < (unsigned)g.P) atomicSub(g.refs + p, 1);
        g.table[(size_t)s * g.C + c] = -1;
      }
      if (lane == 0) g.lens[s] = 0;
    }
    if (lane == 0) done[i] = yes;
  }
}

// Sequence dst[i], which is empty, becomes what src[i] is: it names the same pages, but for a last one that is not full: that one
// is to be copied, copies[i] = (page, its copy) (else -1, -1).
__global__ __launch_bounds__(PGS_THREADS) void k_pages_fork(PagesView g, const int* __restrict__ src, const int* __restrict__ dst, int n,
                                                            int* __restrict__ done, int2* __restrict__ copies) {
  __shared__ PgsScan scan;
  __shared__ int to_s[PGS_THREADS], src_s[PGS_THREADS], dst_s[PGS_THREADS], len_s[PGS_THREADS], ids_s[PGS_LDS_IDS], owner_s[PGS_LDS_OWNERS];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  PgsRefs first;
  first.load(g, 0);
  int from, into, len;                                       // of request i0 + tid: its sequences, the length of the one (-1: not this request)
  auto read = [&](int i) {
    from = src[min(i, n - 1)], into = dst[min(i, n - 1)];
    const bool named = i < n && (unsigned)from < (unsigned)g.S && (unsigned)into < (unsigned)g.S && from != into;
    const int there = g.lens[named ? into : 0], tokens = g.lens[named ? from : 0];
    len = named && there == 0 ? min(max(tokens, 0), g.C * 64) : -1;
  };
  const bool one = n <= PGS_THREADS;                         // (all requests at once: they are read once)
  read(tid);
  int* owner = pgs_owners_clear(g, owner_s, n);
  for (int i = tid; i < n; i += PGS_THREADS) {
    if (!one) read(i);
    if (len >= 0) atomicMin(owner + into, i);
  }
  __syncthreads();
  int want = 0;
  for (int i0 = 0; i0 < n; i0 += PGS_THREADS) {
    const int i = i0 + tid;
    int total;
    if (!one) read(i);
    if (len >= 0 && owner[into] != i) len = -1;
    if (!one && i < n) g.info[i] = len;                      // (before the call: what is given below changes lens)
    const int part = len >= 0 && len % 64 != 0;
    (void)pgs_scan(part, total, scan);
    want += total;
  }
  const PgsList ids{ids_s, g.ids};
  const int found = pgs_collect(g, first, 0, g.P, min(want, g.P), ids, scan, [](int r) { return r == 0; });
  int given = 0;
  for (int i0 = 0; i0 < n; i0 += PGS_THREADS) {
    const int i = i0 + tid;
    if (!one) from = src[min(i, n - 1)], into = dst[min(i, n - 1)], len = i < n ? g.info[i] : -1;
    const int part = len >= 0 && len % 64 != 0;
    int total;
    const int upto = given + pgs_scan(part, total, scan);
    const bool yes = len >= 0 && (!part || upto <= found);
    given += total;
    const int to = yes ? (part ? ids.get(upto - 1) : -2) : -1;   // the copy's page, -2: none needed, -1: not this one
    to_s[tid] = to, len_s[tid] = len, src_s[tid] = from, dst_s[tid] = into;
    if (i < n) {
      done[i] = yes;
      copies[i] = yes && part ? make_int2(g.table[(size_t)from * g.C + len / 64], to) : make_int2(-1, -1);
    }
    __syncthreads();
    for (int u = wv; u < PGS_THREADS && i0 + u < n; u += PGS_THREADS / 64) {
      const int to = to_s[u];
      if (to == -1) continue;
      const int a = src_s[u], d = dst_s[u], full = len_s[u] / 64;
      for (int c = lane; c < g.C; c += 64) {
        int p = -1;
        if (c < full) {
          p = g.table[(size_t)a * g.C + c];
          if ((unsigned)p < (unsigned)g.P) atomicAdd(g.refs + p, 1);
        } else if (c == full && to >= 0) {
          p = to;
          g.refs[p] = 1;
        }
        g.table[(size_t)d * g.C + c] = p;
      }
      if (lane == 0) g.lens[d] = len_s[u];
    }
    __syncthreads();
  }
}

// The used pages take the places 0 .. used - 1: those behind go, in their order, to the free places in front.  ids[p] = where
// page p goes (or p), copies[i] = (from, to), then (-1, -1).
__global__ __launch_bounds__(PGS_THREADS) void k_pages_compact(PagesView g, int2* __restrict__ copies, int n_copies) {
  __shared__ PgsScan scan;
  __shared__ int to_s[PGS_LDS_IDS], from_s[PGS_LDS_IDS];
  const int tid = threadIdx.x;
  PgsRefs first;
  first.load(g, 0);
  int used = 0;
  for (int p0 = 0; p0 < g.P; p0 += PGS_EACH * PGS_THREADS) {
    PgsRefs x = first;
    if (p0) x.load(g, p0);
    int n = 0, total;
#pragma unroll
    for (int u = 0; u < PGS_EACH; ++u) n += p0 + PGS_EACH * tid + u < g.P && x.r[u] > 0;
    (void)pgs_scan(n, total, scan);
    used += total;
  }
  // holes in front, used pages behind
  const PgsList to{to_s, g.ids}, from{from_s, g.ids + g.P};
  const int moves = pgs_collect(g, first, 0, used, n_copies, to, scan, [](int r) { return r <= 0; });
  (void)pgs_collect(g, first, used, g.P, n_copies, from, scan, [](int r) { return r > 0; });
  for (int i = tid; i < n_copies; i += PGS_THREADS) copies[i] = i < moves ? make_int2(from.get(i), to.get(i)) : make_int2(-1, -1);
  __syncthreads();
  for (int p = tid; p < g.P; p += PGS_THREADS) g.ids[p] = p;
  __syncthreads();
  for (int i = tid; i < moves; i += PGS_THREADS) {
    const int2 m = copies[i];
    g.ids[m.x] = m.y;
    g.refs[m.y] = g.refs[m.x];
    g.refs[m.x] = 0;
  }
}
// grid ceil(S C / 256), block 256
__global__ __launch_bounds__(256) void k_pages_rename(PagesView g) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)g.S * g.C) return;
  const int p = g.table[i];
  if ((unsigned)p < (unsigned)g.P) g.table[i] = g.ids[p];
}

// ---- copying ------------------------------------------------------------------------------------
constexpr int PGC_CACHES = 64;           // caches of a launch
constexpr int PGC_PIECE = 16384;         // bytes of a page that a workgroup copies
struct PagesCopyArgs {
  unsigned char* k[PGC_CACHES];
  unsigned char* v[PGC_CACHES];
  float* k_scale[PGC_CACHES];
  float* v_scale[PGC_CACHES];
  int k_bytes[PGC_CACHES], v_bytes[PGC_CACHES];   // of a page (multiples of 16)
  int Hkv[PGC_CACHES];
  const int2* copies;
  int n_pages;
};
// grid (copies, pieces of the largest page, caches), block 256: 16 KB of a page's K and V, read and written once (1.04 GB in 200 us, a large copy's rate); the first piece takes the scales along.
__global__ __launch_bounds__(256) void k_pages_copy(PagesCopyArgs a) {
  const int2 m = a.copies[blockIdx.x];
  if ((unsigned)m.x >= (unsigned)a.n_pages || (unsigned)m.y >= (unsigned)a.n_pages) return;
  const int l = blockIdx.z, tid = threadIdx.x;
  const size_t kb = a.k_bytes[l], vb = a.v_bytes[l];
  typedef unsigned int c_u32x4 __attribute__((ext_vector_type(4)));
  constexpr int N = PGC_PIECE / 4096;
  const size_t at0 = (size_t)blockIdx.y * PGC_PIECE + tid * 16;
  c_u32x4 x[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const size_t at = at0 + u * 4096;
    if (at < kb) x[u] = *(const c_u32x4*)(a.k[l] + m.x * kb + at);
    else if (at < kb + vb) x[u] = *(const c_u32x4*)(a.v[l] + m.x * vb + (at - kb));
  }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const size_t at = at0 + u * 4096;
    if (at < kb) *(c_u32x4*)(a.k[l] + m.y * kb + at) = x[u];
    else if (at < kb + vb) *(c_u32x4*)(a.v[l] + m.y * vb + (at - kb)) = x[u];
  }
  if (blockIdx.y == 0)
    for (int h = tid; h < a.Hkv[l]; h += 256) {
      if (kb) a.k_scale[l][(size_t)m.y * a.Hkv[l] + h] = a.k_scale[l][(size_t)m.x * a.Hkv[l] + h];
      a.v_scale[l][(size_t)m.y * a.Hkv[l] + h] = a.v_scale[l][(size_t)m.x * a.Hkv[l] + h];
    }
}

}  // namespace lisa
