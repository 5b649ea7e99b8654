// Decode steps over the paged 8-bit cache on the matrix cores (kernels_cache8_mfma.h): which calls take that way, their
// workspace, their launches.  LISA_PART 0 .. 3: the scores kernels (ADD and CONCAT, ReLU and SiLU); 4, 5: softmax and P V by format; 6: the rest.
#include "host.h"
#include "kernels_cache8_mfma.h"

namespace lisa {

namespace {
template <int HBI, int FS, int HBO, int ACT, int MODE, int KS, int KVT>
int launch_scores_t(const lisa_desc* d, Cache8ScoresArgs a, hipStream_t st) {
  const int lds = cache8_scores_lds(d->H, KS, MODE == 0 ? 0 : MfmaFfn<HBI, FS, HBO, ACT>::kStageBytes);
  auto kern = k_cache8_scores_mfma<HBI, FS, HBO, ACT, MODE, KS, KVT>;
  if (lds > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return hip_fail(e);
  }
  StageScope prof("k_cache8_scores_mfma", st);
  // Pages per workgroup: as few as leave no more workgroups than the card holds at once (queries and weights are staged once per workgroup, and
  // a second round of workgroups would be as long as the first).  64 sequences of up to 4097 tokens, 32 heads, us for the layer: ADD 192, with
  // half as many pages 195, with twice as many 221.
  constexpr int PER_CU = MODE < 2 && KVT == 1 && HBI <= 2 ? 3 : 2;   // by registers
  const int pages = (d->Lk + PG_TOK - 1) / PG_TOK, room = std::max(1, kComputeUnits * std::min(PER_CU, 160 * 1024 / lds) / d->B);   // workgroups per sequence
  a.n_pages = std::min(64, (pages + room - 1) / room);
  kern<<<dim3((pages + a.n_pages - 1) / a.n_pages, d->B), 256, lds, st>>>(a);
  return check_launch();
}
template <int HBI, int FS, int HBO, int ACT, int MODE>
int launch_scores_ks(const lisa_desc* d, const Cache8ScoresArgs& a, hipStream_t st) {
  if (a.c.w > 32) return launch_scores_t<HBI, FS, HBO, ACT, MODE, 2, 4>(d, a, st);
  return d->H / d->Hkv % 4 == 0 ? launch_scores_t<HBI, FS, HBO, ACT, MODE, 1, 1>(d, a, st) : launch_scores_t<HBI, FS, HBO, ACT, MODE, 1, 4>(d, a, st);
}
template <int HB, int ACT>
int launch_add_fs(const lisa_desc* d, const Cache8ScoresArgs& a, hipStream_t st) {
  switch ((a.F + 31) / 32) {
    case 1: return launch_scores_ks<HB, 1, HB, ACT, 1>(d, a, st);
    case 2: return launch_scores_ks<HB, 2, HB, ACT, 1>(d, a, st);
    case 3: return launch_scores_ks<HB, 3, HB, ACT, 1>(d, a, st);
    default: return launch_scores_ks<HB, 4, HB, ACT, 1>(d, a, st);
  }
}
template <int HBI, int HBO, int ACT>
int launch_concat_fs(const lisa_desc* d, const Cache8ScoresArgs& a, hipStream_t st) {
  if (a.F <= 64) return launch_scores_ks<HBI, 2, HBO, ACT, 2>(d, a, st);
  if (a.F <= 128) return launch_scores_ks<HBI, 4, HBO, ACT, 2>(d, a, st);
  return launch_scores_ks<HBI, 8, HBO, ACT, 2>(d, a, st);
}
}  // namespace

template <int ACT>
int launch_cache8_add(const lisa_desc* d, const Cache8ScoresArgs& a, hipStream_t st);
template <int ACT>
int launch_cache8_concat(const lisa_desc* d, const Cache8ScoresArgs& a, hipStream_t st);
template <int FMT>
int launch_cache8_pv(const lisa_desc* d, int mode, int wide, const Cache8PvArgs& a, hipStream_t st);

#if LISA_PART <= 1
template <int ACT>
int launch_cache8_add(const lisa_desc* d, const Cache8ScoresArgs& a, hipStream_t st) {
  switch ((d->H + 15) / 16) {
    case 1: return launch_add_fs<1, ACT>(d, a, st);
    case 2: return launch_add_fs<2, ACT>(d, a, st);
    case 3: return launch_add_fs<3, ACT>(d, a, st);
    default: return launch_add_fs<4, ACT>(d, a, st);
  }
}
template int launch_cache8_add<LISA_PART>(const lisa_desc*, const Cache8ScoresArgs&, hipStream_t);
#elif LISA_PART <= 3
template <int ACT>
int launch_cache8_concat(const lisa_desc* d, const Cache8ScoresArgs& a, hipStream_t st) {
  return d->H <= 16 ? launch_concat_fs<2, 1, ACT>(d, a, st) : d->H <= 32 ? launch_concat_fs<4, 2, ACT>(d, a, st) : launch_concat_fs<6, 3, ACT>(d, a, st);
}
template int launch_cache8_concat<LISA_PART - 2>(const lisa_desc*, const Cache8ScoresArgs&, hipStream_t);
#elif LISA_PART <= 5
namespace {
template <int FMT, int DK, int MODE, int GT, int GH>
int launch_pv_nw(const lisa_desc* d, int wide, const Cache8PvArgs& a, hipStream_t st) {
  const dim3 grid(d->Hkv * a.chunks * a.f_parts, a.n_span, d->B);
  StageScope prof("k_cache8_pv", st);
  constexpr bool EIGHT = MODE > 0 && GT == 1;                // (pv_geom)
  if (EIGHT && wide) k_cache8_pv<FMT, DK, MODE, GT, GH, EIGHT ? 8 : 4><<<grid, 512, 0, st>>>(a);
  else k_cache8_pv<FMT, DK, MODE, GT, GH, 4><<<grid, 256, 0, st>>>(a);
  return check_launch();
}
template <int FMT, int DK, int MODE>
int launch_pv_heads(const lisa_desc* d, int wide, const Cache8PvArgs& a, hipStream_t st) {
  const int group = d->H / d->Hkv;
  if (group == 1) return launch_pv_nw<FMT, DK, MODE, 1, 1>(d, wide, a, st);
  if (group <= 4) return launch_pv_nw<FMT, DK, MODE, 1, 4>(d, wide, a, st);
  return launch_pv_nw<FMT, DK, MODE, 2, 4>(d, wide, a, st);
}
template <int FMT, int DK>
int launch_pv_mode(const lisa_desc* d, int mode, int wide, const Cache8PvArgs& a, hipStream_t st) {
  return mode == 0   ? launch_pv_heads<FMT, DK, 0>(d, wide, a, st)
         : mode == 1 ? launch_pv_heads<FMT, DK, 1>(d, wide, a, st)
                     : launch_pv_heads<FMT, DK, 2>(d, wide, a, st);
}
}  // namespace
template <int FMT>
int launch_cache8_pv(const lisa_desc* d, int mode, int wide, const Cache8PvArgs& a, hipStream_t st) {
  return d->d_k / a.f_parts == 128 ? launch_pv_mode<FMT, 128>(d, mode, wide, a, st) : launch_pv_mode<FMT, 64>(d, mode, wide, a, st);
}
template int launch_cache8_pv<LISA_PART - 4>(const lisa_desc*, int, int, const Cache8PvArgs&, hipStream_t);
#else

namespace {

// The module that the scores kernel runs: a single layer y = W^T x is the ReLU network [W, -W], [I; -I] (stage_ffn).
struct Module {
  int Din, F, act, mix;
};
Module module_of(const lisa_desc* d) {
  Module m;
  m.mix = d->mix;
  m.Din = d->mix == LISA_MIX_CONCAT ? 2 * d->H : d->H;
  m.F = d->act == LISA_ACT_SINGLE ? 2 * d->H : d->F;
  m.act = d->act == LISA_ACT_SILU ? 1 : 0;
  return m;
}
// Softmax and P V: what a workgroup spends before its first page and after its last (page numbers, scales and queries; merging its waves) is
// some five pages' time, so a (sequence, kv head) is one workgroup's work where that makes 256 of them, one per compute unit; else it
// is split until there are, more than 16 pages into eights at the smallest (a launch more, some 3 us; LiSA, one sequence of 3000 tokens, 8 kv heads:
// 16.0 us, unsplit 21.5; of 1000: 15.9 and 14.7).  Eight waves for LiSA layers: a stream of V runs best with few of them per compute unit
// (64 sequences of up to 4097 tokens, 32 heads: 192 us for the layer, 223 with four such workgroups of four waves per compute unit).
// Four for standard layers (fewer leave their registers room; 32 sequences of up to 8192, 8 kv heads: 76 us, 85 at eight spans instead of one),
// where a wave has more than four heads (256 registers do not hold them with eight) and where several workgroups per compute unit with 32
// pages at most follow one another (64 sequences of up to 500 tokens, 32 heads: 35 us, with eight 43; at 2500 129 and 126).
// Features are dealt to two workgroups, which needs no merging, where that spares a split or none is made anyway (LiSA, 16 sequences of up to 1000
// tokens, 8 kv heads: 14.6 us, 15.7 without; with splits it only adds workgroups: 4 of 3000 17.4 and 17.0).
struct PvGeom {
  int wide, span_pages, n_span, chunks, f_parts;
};
PvGeom pv_geom(const lisa_desc* d, bool lisa_layer) {
  const int group = d->H / d->Hkv, n_pages = std::max((d->Lk + PG_TOK - 1) / PG_TOK, 1);
  PvGeom g;
  g.chunks = group <= 4 ? 1 : (group + 7) / 8;
  long long base = (long long)d->B * d->Hkv * g.chunks;
  g.f_parts = lisa_layer && d->d_k == 128 && base <= 128 && (n_pages <= 16 || base == 128) ? 2 : 1;
  base *= g.f_parts;
  g.wide = lisa_layer && group <= 4 && (base < 512 || n_pages > 32);
  const int waves = g.wide ? 8 : 4;
  const int spans = n_pages <= 16 ? 1 : (int)std::min<long long>((256 + base - 1) / base, (n_pages + 7) / 8);
  g.span_pages = std::min((int)round_up((n_pages + spans - 1) / spans, waves), 64 * waves);
  g.n_span = (n_pages + g.span_pages - 1) / g.span_pages;
  return g;
}

struct Ws {
  size_t s, part_o, part_ml, total;
  int Lp;
};
Ws ws_of(const lisa_desc* d, bool lisa_layer) {
  const PvGeom g = pv_geom(d, lisa_layer);
  Ws w{};
  w.Lp = (d->Lk + PG_TOK - 1) / PG_TOK * PG_TOK;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t r = at;
    at = round_up(at + bytes, 256);
    return r;
  };
  const size_t parts = g.n_span > 1 ? (size_t)d->B * g.n_span * d->H : 0;
  w.part_o = take(parts * d->d_k * sizeof(float));
  w.part_ml = take(parts * 2 * sizeof(float));
  if (lisa_layer && d->mix != LISA_MIX_SHARE) w.s = take((size_t)d->B * d->H * w.Lp * sizeof(float));
  w.total = std::max<size_t>(at, 256);
  return w;
}

}  // namespace

bool cache8_fast_ok(const lisa_desc* d, bool lisa_layer) {
  if (d->dtype != LISA_BF16 || (d->d_k != 64 && d->d_k != 128)) return false;
  if ((long long)(d->H / d->Hkv + 7) / 8 * d->Hkv > 65535 || d->Lk > 1 << 29) return false;   // (the grid: spans of 256 pages at the most)
  if (!lisa_layer || d->mix == LISA_MIX_SHARE) return true;
  if (d->r > 64 || d->H > 64 || (long long)d->H * d->Lk >= 1LL << 30) return false;   // (32-bit offsets in a sequence's score rows)
  if (d->mix == LISA_MIX_PLUS) return true;
  const Module m = module_of(d);
  return d->mix == LISA_MIX_CONCAT ? d->H <= 48 && m.F <= 256 : m.F <= 128;
}

size_t cache8_fast_bytes(const lisa_desc* d, bool lisa_layer) { return ws_of(d, lisa_layer).total; }

int run_cache8_fast(const lisa_desc* d, bool lisa_layer, int fmt, const Cache8View& c, const void* q, const void* prev, const void* w1,
                    const void* w2, float scale, void* row, void* out, void* workspace, hipStream_t st) {
  const Ws w = ws_of(d, lisa_layer);
  const PvGeom g = pv_geom(d, lisa_layer);
  char* ws = (char*)workspace;
  const bool share = lisa_layer && d->mix == LISA_MIX_SHARE;
  if (lisa_layer && !share) {
    Cache8ScoresArgs a{};
    a.c = c;
    a.q = (const bf16_t*)q;
    a.prev = (const half_t*)prev;
    a.row = (half_t*)row;
    a.s = (float*)(ws + w.s);
    a.H = d->H;
    a.Lk = d->Lk;
    a.Lp = w.Lp;
    a.fmt = fmt;
    a.scale = scale;
    int rc;
    if (d->mix == LISA_MIX_PLUS) {
      rc = launch_scores_ks<1, 1, 1, 0, 0>(d, a, st);
    } else {
      const Module m = module_of(d);
      a.w1 = (const bf16_t*)w1;
      a.w2 = d->act == LISA_ACT_SINGLE ? nullptr : (const bf16_t*)w2;
      a.F = m.F;
      rc = d->mix == LISA_MIX_CONCAT ? (m.act ? launch_cache8_concat<1>(d, a, st) : launch_cache8_concat<0>(d, a, st))
                                     : (m.act ? launch_cache8_add<1>(d, a, st) : launch_cache8_add<0>(d, a, st));
    }
    if (rc) return rc;
  }
  Cache8PvArgs p{};
  p.c = c;
  p.q = (const bf16_t*)q;
  p.s = (const float*)(ws + w.s);
  p.prev = (const half_t*)prev;
  p.row = lisa_layer && !share ? nullptr : (half_t*)row;
  p.out = out;
  p.part_o = (float*)(ws + w.part_o);
  p.part_ml = (float*)(ws + w.part_ml);
  p.H = d->H;
  p.Lk = d->Lk;
  p.Lp = w.Lp;
  p.n_span = g.n_span;
  p.span_pages = g.span_pages;
  p.chunks = g.chunks;
  p.f_parts = g.f_parts;
  p.out_f32 = d->out_f32;
  p.scale = scale;
  const int mode = !lisa_layer ? 0 : share ? 2 : 1;
  int rc = fmt ? launch_cache8_pv<1>(d, mode, g.wide, p, st) : launch_cache8_pv<0>(d, mode, g.wide, p, st);
  if (rc) return rc;
  if (g.n_span > 1) {
    StageScope prof("k_cache8_combine", st);
    auto kern = d->d_k == 128 ? k_cache8_combine<128> : k_cache8_combine<64>;
    kern<<<dim3(d->H, d->B), d->d_k, 0, st>>>(p.part_o, p.part_ml, c.lens, out, d->H, d->Lk, g.n_span, g.span_pages * PG_TOK, d->out_f32);
    rc = check_launch();
  }
  if (rc == LISA_OK) note_path("decode8");
  return rc;
}
#endif

}  // namespace lisa
