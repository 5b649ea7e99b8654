// C ABI of the paged 8-bit cache: argument validation (host only, before any HIP call), workspace accounting and dispatch.
#include "host.h"
#include "kernels_cache8.h"
#include "kernels_pages.h"

using namespace lisa;

namespace lisa {
// launch_cache8.hip
bool cache8_fast_ok(const lisa_desc* d, bool lisa_layer);
size_t cache8_fast_bytes(const lisa_desc* d, bool lisa_layer);
int run_cache8_fast(const lisa_desc* d, bool lisa_layer, int fmt, const Cache8View& c, const void* q, const void* prev, const void* w1,
                    const void* w2, float scale, void* row, void* out, void* workspace, hipStream_t st);
}  // namespace lisa

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

constexpr int kMaxWidth = 256;           // key and value rows (k_cache8_softmax_v: a thread per feature)
constexpr int kMaxPages = 1 << 20;
constexpr int kMaxGridYZ = 65535;

int check_cache(const lisa_cache8* c) {
  if (!c) return LISA_ERR_NULL;
  if (c->format != LISA_CACHE_INT8 && c->format != LISA_CACHE_E4M3) return LISA_ERR_UNSUPPORTED;
  if (c->n_pages <= 0 || c->max_pages <= 0 || c->Hkv <= 0 || c->width < 0 || c->d_k <= 0) return LISA_ERR_SHAPE;
  if (c->n_pages > kMaxPages || c->width > kMaxWidth || c->d_k > kMaxWidth || c->Hkv > kMaxGridYZ || c->max_pages > (1 << 24))
    return LISA_ERR_UNSUPPORTED;
  if (!c->v || !c->v_scale || (c->width && (!c->k || !c->k_scale))) return LISA_ERR_NULL;
  if (!aligned16(c->v) || !aligned16(c->k) || !aligned4(c->v_scale) || !aligned4(c->k_scale)) return LISA_ERR_ALIGN;
  return LISA_OK;
}
int check_sequences(const lisa_cache8* c) {
  if (!c->table || !c->lens) return LISA_ERR_NULL;
  return aligned4(c->table) && aligned4(c->lens) ? LISA_OK : LISA_ERR_ALIGN;
}

Cache8View view(const lisa_cache8* c) {
  Cache8View v;
  v.k = (unsigned char*)c->k;
  v.k_scale = c->k_scale;
  v.v = (unsigned char*)c->v;
  v.v_scale = c->v_scale;
  v.table = c->table;
  v.lens = c->lens;
  v.n_pages = c->n_pages;
  v.max_pages = c->max_pages;
  v.Hkv = c->Hkv;
  v.w = c->width;
  v.w8 = (c->width + 7) / 8 * 8;
  v.dk = c->d_k;
  return v;
}

// Descriptor of a decode step over an 8-bit cache.
int check_decode8(const lisa_desc* d, bool lisa_layer) {
  if (!d) return LISA_ERR_NULL;
  lisa_desc t = *d;
  t.causal = 0;                                              // (one query row sees all tokens)
  int rc = lisa_layer ? check_lisa_desc(&t) : check_common_desc(&t);
  if (rc) return rc;
  if (d->Lq != 1) return LISA_ERR_SHAPE;
  return d->score_tiled ? LISA_ERR_UNSUPPORTED : LISA_OK;    // a decode step hands over score rows
}
int check_match(const lisa_desc* d, const lisa_cache8* c, int width) {
  if (c->Hkv != d->Hkv || c->d_k != d->d_k || (width >= 0 && c->width != width)) return LISA_ERR_SHAPE;
  return d->Lk > (long long)c->max_pages * LISA_PAGE_TOKENS ? LISA_ERR_SHAPE : LISA_OK;
}

size_t generic_bytes(const lisa_desc* d) { return round_up((size_t)d->B * d->H * d->Lk * sizeof(float), 256); }

template <typename T, typename S, int FMT>
int run_generic(const lisa_desc* d, const Cache8View& c, const void* q, const void* prev, const void* w1, const void* w2, int mix,
                float scale, void* scores, void* out, void* workspace, hipStream_t st) {
  float* exact = (float*)workspace;
  const int Din = mix == LISA_MIX_CONCAT ? 2 * d->H : d->H;
  const size_t lds = mix <= LISA_MIX_CONCAT ? (size_t)(Din + d->F + d->H) * 64 * sizeof(float) : 0;
  auto kern = k_cache8_scores<T, S, FMT>;
  if (lds > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return hip_fail(e);
  }
  {
    StageScope prof("k_cache8_scores", st);
    kern<<<dim3((d->Lk + 63) / 64, d->B), 256, lds, st>>>(c, (const T*)q, (const S*)prev, (const T*)w1, (const T*)w2, (S*)scores, exact,
                                                          d->H, d->Lk, d->F, mix, d->act, scale);
    if (int rc = check_launch()) return rc;
  }
  StageScope prof("k_cache8_softmax_v", st);
  const dim3 grid(d->H, d->B);
  if (d->out_f32) k_cache8_softmax_v<T, float, FMT><<<grid, 256, 0, st>>>(c, exact, (float*)out, d->H, d->Lk);
  else k_cache8_softmax_v<T, T, FMT><<<grid, 256, 0, st>>>(c, exact, (T*)out, d->H, d->Lk);
  const int rc = check_launch();
  if (rc == LISA_OK) note_path("decode8_generic");
  return rc;
}

int run_decode8(const lisa_desc* d, const lisa_cache8* cache, const void* q, const void* prev, const void* w1, const void* w2, int mix,
                float scale, void* scores, void* out, void* workspace, hipStream_t st) {
  const Cache8View c = view(cache);
  const bool e4m3 = cache->format == LISA_CACHE_E4M3, lisa_layer = mix != 4;
  if (cache8_fast_ok(d, lisa_layer))
    return run_cache8_fast(d, lisa_layer, e4m3, c, q, prev, w1, w2, scale, scores, out, workspace, st);
  auto run = d->dtype == LISA_F32 ? (e4m3 ? run_generic<float, float, 1> : run_generic<float, float, 0>)
                                  : (e4m3 ? run_generic<bf16_t, half_t, 1> : run_generic<bf16_t, half_t, 0>);
  return run(d, c, q, prev, w1, w2, mix, scale, scores, out, workspace, st);
}

template <typename T>
void launch_append(const Cache8View& c, bool e4m3, dim3 grid, const void* k_new, const void* v_new, const int32_t* counts, int L, hipStream_t st) {
  if (L == 1) {
    auto kern = e4m3 ? k_cache8_append_token<T, 1> : k_cache8_append_token<T, 0>;
    kern<<<dim3((c.Hkv + 3) / 4, grid.z), 256, 0, st>>>(c, (const T*)k_new, (const T*)v_new, counts);
    return;
  }
  const bool wide = c.w > 128 || c.dk > 128;
  auto kern = e4m3 ? (wide ? k_cache8_append<T, 1, true> : k_cache8_append<T, 1, false>)
                   : (wide ? k_cache8_append<T, 0, true> : k_cache8_append<T, 0, false>);
  kern<<<grid, 256, 0, st>>>(c, (const T*)k_new, (const T*)v_new, counts, L);
}

// ---- pages ------------------------------------------------------------------------------------
int check_pages(const lisa_pages* p) {
  if (!p) return LISA_ERR_NULL;
  if (p->n_pages <= 0 || p->n_seqs <= 0 || p->max_pages <= 0 || p->reserved != 0) return LISA_ERR_SHAPE;
  if (p->n_pages > kMaxPages || p->max_pages > (1 << 24) || (long long)p->n_seqs * p->max_pages > (1LL << 31) - 256)
    return LISA_ERR_UNSUPPORTED;
  if (!p->table || !p->lens || !p->refs) return LISA_ERR_NULL;
  return aligned4(p->table) && aligned4(p->lens) && aligned4(p->refs) ? LISA_OK : LISA_ERR_ALIGN;
}
int pages_view(const lisa_pages* p, void* workspace, size_t workspace_bytes, PagesView* g) {
  int rc = check_pages(p);
  if (rc) return rc;
  if (workspace && !aligned16(workspace)) return LISA_ERR_ALIGN;
  if (!workspace || workspace_bytes < lisa_pages_workspace_bytes(p)) return LISA_ERR_WORKSPACE;
  g->table = p->table;
  g->lens = p->lens;
  g->refs = p->refs;
  g->P = p->n_pages;
  g->S = p->n_seqs;
  g->C = p->max_pages;
  g->owner = (int*)workspace;
  g->info = g->owner + p->n_seqs;
  g->ids = g->info + p->n_seqs;
  return LISA_OK;
}
int pages_done() {
  const int rc = check_launch();
  if (rc == LISA_OK) note_path("pages");
  return rc;
}

}  // namespace

namespace lisa {
size_t decode8_bytes(const lisa_desc* d, bool lisa_layer) {
  if (check_decode8(d, lisa_layer) != LISA_OK) return 0;
  return cache8_fast_ok(d, lisa_layer) ? cache8_fast_bytes(d, lisa_layer) : generic_bytes(d);
}
}  // namespace lisa

extern "C" {

int lisa_cache8_append(const lisa_desc* d, const lisa_cache8* cache, const void* k_new, const void* v_new,
                       const int32_t* counts, void* hip_stream) {
  if (!d) return LISA_ERR_NULL;
  int rc = check_cache(cache);
  if (rc) return rc;
  rc = check_sequences(cache);
  if (rc) return rc;
  if (d->dtype != LISA_F32 && d->dtype != LISA_BF16) return LISA_ERR_UNSUPPORTED;
  if (d->B <= 0 || d->Lq <= 0 || d->Hkv != cache->Hkv || d->r != cache->width || d->d_k != cache->d_k) return LISA_ERR_SHAPE;
  if (d->B > kMaxGridYZ) return LISA_ERR_UNSUPPORTED;
  if (!v_new || (cache->width && !k_new)) return LISA_ERR_NULL;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned4(counts)) return LISA_ERR_ALIGN;
  hipStream_t st = (hipStream_t)hip_stream;
  const Cache8View c = view(cache);
  const dim3 grid((unsigned)(((long long)d->Lq + 126) / 64), d->Hkv, d->B);
  StageScope prof("k_cache8_append", st);
  const bool e4m3 = cache->format == LISA_CACHE_E4M3;
  if (d->dtype == LISA_F32) launch_append<float>(c, e4m3, grid, k_new, v_new, counts, d->Lq, st);
  else launch_append<bf16_t>(c, e4m3, grid, k_new, v_new, counts, d->Lq, st);
  rc = check_launch();
  if (rc == LISA_OK) note_path("cache8_append");
  return rc;
}

int lisa_attn_decode8(const lisa_desc* d, const lisa_cache8* cache, const void* q_lr, const void* score_row_prev, const void* w1,
                      const void* w2, void* out, void* score_row_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_decode8(d, true);
  if (rc) return rc;
  rc = check_cache(cache);
  if (rc) return rc;
  rc = check_sequences(cache);
  if (rc) return rc;
  const bool delta = d->mix != LISA_MIX_SHARE, ffn = d->mix == LISA_MIX_ADD || d->mix == LISA_MIX_CONCAT;
  rc = check_match(d, cache, delta ? d->r : -1);
  if (rc) return rc;
  if (!score_row_prev || !out || (delta && !q_lr)) return LISA_ERR_NULL;
  if (ffn && (!w1 || (d->act != LISA_ACT_SINGLE && !w2))) return LISA_ERR_NULL;
  if (d->write_scores && !score_row_out) return LISA_ERR_NULL;
  if (d->write_scores && score_row_out == score_row_prev) return LISA_ERR_SHAPE;
  const void* ptrs[] = {q_lr, score_row_prev, w1, w2, out, score_row_out, workspace};
  for (const void* p : ptrs)
    if (!aligned16(p)) return LISA_ERR_ALIGN;
  if (!workspace || workspace_bytes < lisa_workspace_bytes(d, LISA_WS_DECODE8)) return LISA_ERR_WORKSPACE;
  return run_decode8(d, cache, q_lr, score_row_prev, w1, w2, d->mix, delta ? pick_scale(d->delta_scale, d->r) : 0.f,
                     d->write_scores ? score_row_out : nullptr, out, workspace, (hipStream_t)hip_stream);
}

int std_attn_decode8(const lisa_desc* d, const lisa_cache8* cache, const void* q, void* score_row_out, void* out, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
  int rc = check_decode8(d, false);
  if (rc) return rc;
  rc = check_cache(cache);
  if (rc) return rc;
  rc = check_sequences(cache);
  if (rc) return rc;
  rc = check_match(d, cache, d->d_k);
  if (rc) return rc;
  if (!q || !out) return LISA_ERR_NULL;
  const void* ptrs[] = {q, out, score_row_out, workspace};
  for (const void* p : ptrs)
    if (!aligned16(p)) return LISA_ERR_ALIGN;
  if (!workspace || workspace_bytes < lisa_workspace_bytes(d, LISA_WS_STD_DECODE8)) return LISA_ERR_WORKSPACE;
  return run_decode8(d, cache, q, nullptr, nullptr, nullptr, 4, pick_scale(d->std_scale, d->d_k), score_row_out, out, workspace,
                     (hipStream_t)hip_stream);
}

size_t lisa_pages_workspace_bytes(const lisa_pages* p) {
  return check_pages(p) == LISA_OK ? round_up(((size_t)p->n_pages + p->n_seqs) * 2 * sizeof(int), 256) : 0;
}

int lisa_pages_grow(const lisa_pages* pages, const int32_t* add, int32_t* done, void* workspace, size_t workspace_bytes,
                    void* hip_stream) {
  PagesView g;
  int rc = pages_view(pages, workspace, workspace_bytes, &g);
  if (rc) return rc;
  if (!add || !done) return LISA_ERR_NULL;
  if (!aligned4(add) || !aligned4(done)) return LISA_ERR_ALIGN;
  hipStream_t st = (hipStream_t)hip_stream;
  StageScope prof("k_pages_grow", st);
  k_pages_grow<<<1, PGS_THREADS, 0, st>>>(g, add, done);
  return pages_done();
}

int lisa_pages_fork(const lisa_pages* pages, const int32_t* src, const int32_t* dst, int32_t n, int32_t* done, int32_t* copies,
                    void* workspace, size_t workspace_bytes, void* hip_stream) {
  PagesView g;
  int rc = pages_view(pages, workspace, workspace_bytes, &g);
  if (rc) return rc;
  if (!src || !dst || !done || !copies) return LISA_ERR_NULL;
  if (n <= 0 || n > pages->n_seqs) return LISA_ERR_SHAPE;
  if (!aligned4(src) || !aligned4(dst) || !aligned4(done) || (reinterpret_cast<uintptr_t>(copies) & 7u)) return LISA_ERR_ALIGN;
  hipStream_t st = (hipStream_t)hip_stream;
  StageScope prof("k_pages_fork", st);
  k_pages_fork<<<1, PGS_THREADS, 0, st>>>(g, src, dst, n, done, (int2*)copies);
  return pages_done();
}

int lisa_pages_free(const lisa_pages* pages, const int32_t* seqs, int32_t n, int32_t* done, void* workspace, size_t workspace_bytes,
                    void* hip_stream) {
  PagesView g;
  int rc = pages_view(pages, workspace, workspace_bytes, &g);
  if (rc) return rc;
  if (!seqs || !done) return LISA_ERR_NULL;
  if (n <= 0 || n > pages->n_seqs) return LISA_ERR_SHAPE;
  if (!aligned4(seqs) || !aligned4(done)) return LISA_ERR_ALIGN;
  hipStream_t st = (hipStream_t)hip_stream;
  StageScope prof("k_pages_free", st);
  k_pages_free<<<1, PGS_THREADS, 0, st>>>(g, seqs, n, done);
  return pages_done();
}

int lisa_pages_compact(const lisa_pages* pages, int32_t* copies, void* workspace, size_t workspace_bytes, void* hip_stream) {
  PagesView g;
  int rc = pages_view(pages, workspace, workspace_bytes, &g);
  if (rc) return rc;
  const int n_copies = pages->n_pages / 2;
  if (!copies && n_copies) return LISA_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(copies) & 7u) return LISA_ERR_ALIGN;
  hipStream_t st = (hipStream_t)hip_stream;
  {
    StageScope prof("k_pages_compact", st);
    k_pages_compact<<<1, PGS_THREADS, 0, st>>>(g, (int2*)copies, n_copies);
    rc = check_launch();
    if (rc) return rc;
  }
  StageScope prof("k_pages_rename", st);
  k_pages_rename<<<(unsigned)(((size_t)g.S * g.C + 255) / 256), 256, 0, st>>>(g);
  return pages_done();
}

int lisa_pages_copy(const lisa_cache8* caches, int32_t n_caches, const int32_t* copies, int32_t n_copies, void* hip_stream) {
  if (!caches || !copies) return LISA_ERR_NULL;
  if (n_caches <= 0 || n_copies <= 0) return LISA_ERR_SHAPE;
  for (int i = 0; i < n_caches; ++i) {
    const int rc = check_cache(caches + i);
    if (rc) return rc;
    if (caches[i].n_pages != caches[0].n_pages) return LISA_ERR_SHAPE;
    if ((size_t)caches[i].Hkv * (caches[i].width + 7 + caches[i].d_k) * LISA_PAGE_TOKENS > (size_t)1 << 29) return LISA_ERR_UNSUPPORTED;
  }
  if (reinterpret_cast<uintptr_t>(copies) & 7u) return LISA_ERR_ALIGN;
  hipStream_t st = (hipStream_t)hip_stream;
  StageScope prof("k_pages_copy", st);
  for (int first = 0; first < n_caches; first += PGC_CACHES) {
    const int n = std::min(PGC_CACHES, n_caches - first);
    PagesCopyArgs a{};
    int page = 0;
    for (int i = 0; i < n; ++i) {
      const lisa_cache8& c = caches[first + i];
      a.k[i] = (unsigned char*)c.k;
      a.v[i] = (unsigned char*)c.v;
      a.k_scale[i] = c.k_scale;
      a.v_scale[i] = c.v_scale;
      a.k_bytes[i] = c.Hkv * ((c.width + 7) / 8 * 8) * LISA_PAGE_TOKENS;
      a.v_bytes[i] = c.Hkv * c.d_k * LISA_PAGE_TOKENS;
      a.Hkv[i] = c.Hkv;
      page = std::max(page, a.k_bytes[i] + a.v_bytes[i]);
    }
    a.copies = (const int2*)copies;
    a.n_pages = caches[0].n_pages;
    k_pages_copy<<<dim3(n_copies, (page + PGC_PIECE - 1) / PGC_PIECE, n), 256, 0, st>>>(a);
    const int rc = check_launch();
    if (rc) return rc;
  }
  note_path("pages");
  return LISA_OK;
}

}  // extern "C"
