// Host side of the LM head's other objectives (mst_objective.h): validation, workspace carving, launches.  Part of mst_api.hip,
// whose plans, forward groups and backward orders these calls run with their own kernels for the logits.
#include "../../include/mst_objective.h"

#include <cmath>
#include <type_traits>

namespace {

struct ObjPlan {
  Plan p;
  int K;
  bool few;              // the forward's tiles are TileFew, not the plain forward's
  int n_vt;              // vocabulary tiles of the forward
  // forward workspace: the plain forward's, then
  size_t f_part_few, f_row_loss, f_part_label, f_starts, f_index, f_logit, f_entry_z, f_info, f_total;
  size_t s_rows, s_rows2, s_index, s_at, s_total;      // of `saved`
};

// Up to so many entries a row, tiles of 64 x 64 dlogits put them in themselves: a launch less, 3 us, for which a tile looks through
// the entries of its rows.
constexpr int kPatchEntries = 64;

// See TileFew.  Where tiles of 256 leave a row's pairs to one thread of k_obj_finalize_one and tiles of 64 do not, short hidden sizes are
// slower with these: 128 rows, V = 4000: d = 128 8.0 us with tiles of 256, 9.3; 512 9.9, 10.3; 1536 16.7, 13.9; 4096 30.0, 21.0.
int few_row_tiles(const Plan& p) { return (int)((p.S + TileFew::EB - 1) / TileFew::EB); }
bool use_tile_few(const Plan& p, int K) {
  if (p.S > p.fwd_group_rows || (p.S + TileFew::EB - 1) / TileFew::EB * p.n_vt > kNumCu / 2) return false;
  return K || p.S <= kObjRows || p.d >= 1024 || p.n_vt > kFinOneTiles || p.V <= kFinOneTiles * TileFew::EA;
}

// One workgroup finishes a forward call without a teacher (k_obj_finalize_one).  Whole calls, us, with it and with the two launches of
// longer ones: 256 rows, d = 512, 32 tiles of 64 11.5, 14.3; d = 1024, 63 tiles (16128 pairs) 14.2, 15.9.  Up to 32 pairs a row are one
// thread's: split over two, and joined in LDS, 512 rows of 16 take 11.3 in place of 10.5.
constexpr int64_t kPairsOfOne = 16384;
int finalize_row_bits(int64_t S, int n_vt) {                       // of its threads, 2^row_bits have the first pair of a row each
  if (n_vt <= kFinOneTiles) return 10;
  int bits = 6;
  while (S > int64_t(1) << bits) ++bits;
  return bits;
}
bool one_finalizes(const ObjPlan& o) {
  if (o.K || o.p.S > 1024 || o.p.S > o.p.fwd_group_rows || o.p.S * o.n_vt > kPairsOfOne) return false;
  return o.n_vt <= kFinOneTiles << (10 - finalize_row_bits(o.p.S, o.n_vt));
}

// Byte ranges of a call's arguments: no output may overlap anything else.
struct Ranges {
  struct R { uintptr_t at; size_t bytes; bool out; };
  R r[20];
  int n = 0;
  void add(const void* p, size_t bytes, bool out) {
    if (p) r[n++] = {reinterpret_cast<uintptr_t>(p), bytes, out};
  }
  bool apart() const {
    for (int i = 0; i < n; ++i)
      for (int j = 0; j < i; ++j)
        if ((r[i].out || r[j].out) && r[i].at < r[j].at + r[j].bytes && r[j].at < r[i].at + r[i].bytes) return false;
    return true;
  }
};

// Mini-sequences that the calls make of a call's M: no more than leave each kObjRoom of fp32 logits.  M bounds the memory, and
// below some hundred MB the backward pays for the bound and the chip has no use for it: its launches get too small to fill the
// compute units.  Backward of the plain cross-entropy, us, by mini-sequences: 5003 rows, d = 1544, V = 32003: 2340 with 19 (32 MB), 1757
// with 10, 1452 with 4, 1380 with 3, 1407 with 2, 1552 with 1 (610 MB); 8192, 4096, 128256: 19616 with 31 (129 MB), 19324 with 16, 18694
// with 8, 18593 with 4 (1 GB); 20000, 520, 30000: 3927 with 57 (40 MB), 2300 with 16, 2245 with 4; 3000, 1024, 8000: 340 with 8, 152 with 1.
constexpr int64_t kObjRoom = int64_t(512) << 20;
int32_t fewer_mini_sequences(int64_t S, int64_t d, int64_t V, int32_t M) {
  if (S < 1 || d < 1 || V < 1 || V >= (int64_t(1) << 31) || M < 1 || M > S) return M;      // refused by make_plan
  // never so long that a mini-sequence's rows x d reach 2^30, which make_plan refuses
  const int64_t rows = std::max<int64_t>(1, std::min(kObjRoom / (4 * ((V + 7) / 8 * 8)), ((int64_t(1) << 30) - 1) / d));
  return (int32_t)std::min<int64_t>(M, (S + rows - 1) / rows);
}

// dW of few vocabulary entries and many rows is a few tiles with a long contraction over the rows, which is split then.  The partials
// fit into the half of the workspace that one mini-sequence's dlogits leave; the launch models are those that rank the tiles.  Backward,
// us, without and with: 30000 rows, d = 128, V = 352 114, 46; 65536, 1024, 512 415, 246; 32768, 2048, 384 245, 217; 16384, 512, 1000 132,
// 94; where the models see less than 15 % the launch stays whole (5000, 2048, 256: 53).
void split_dw(Plan* p) {
  if (p->blk_use || p->joint || p->n_chunks != 1) return;
  const double ksteps = (double)((p->C + kBK - 1) / kBK), bytes = 4.0 * (double)(p->V * p->d);
  const double t64 = tiles_of(p->V, p->d, 64), t256 = tiles_of(p->V, p->d, 256);
  double best = 0.85 * (p->small_dw ? small_launch_us(t64, ksteps) : big_launch_us(t256, ksteps));
  const int64_t room = (int64_t)((double)p->b_slot / bytes);
  for (int s = 2; s <= 64 && s <= room && s <= ksteps; ++s) {
    const double per = std::ceil(ksteps / s), sum = 4.0 + (s + 1) * bytes / 4.6e6;
    const double small = small_launch_us(t64 * s, per) + sum, big = big_launch_us(t256 * s, per) + sum;
    if (std::min(small, big) >= best) continue;
    best = std::min(small, big);
    p->dw_per = (int)per * kBK;
    p->dw_split = (int)std::ceil(ksteps / per);
    p->dw_split_small = small < big;
  }
}

mst_status make_obj_plan(int64_t S, int64_t d, int64_t V, int32_t M, int32_t K, ObjPlan* o, int forced = MST_BWD_SCHEDULE_AUTO,
                         bool schedule = false) {
  const mst_status s = make_plan(S, d, V, fewer_mini_sequences(S, d, V, M), &o->p, forced, 0, schedule);
  if (s != MST_OK) return s;
  if (K < 0 || K > MST_MAX_ENTRIES) return MST_ERR_BAD_SHAPE;
  if (K && S * std::max(K, 64) >= int64_t(1) << 32) return MST_ERR_BAD_SHAPE;      // threads of a launch
  o->p.streamed = 0;      // that order stores no dlogits to put the entries into
  if (schedule) split_dw(&o->p);
  o->K = K;
  o->few = use_tile_few(o->p, K);
  o->n_vt = o->few ? (int)((V + TileFew::EA - 1) / TileFew::EA) : o->p.n_vt;
  const size_t rows = (size_t)o->p.fwd_group_rows, k = (size_t)K;
  size_t off = o->p.f_total;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return at; };
  o->f_part_few = o->few ? take((size_t)o->n_vt * rows * 8) : 0;
  o->f_row_loss = take((size_t)S * 8);
  o->f_part_label = K ? take((size_t)o->n_vt * rows * 4) : 0;
  o->f_starts = K && !o->few ? take((size_t)(o->n_vt + 1) * rows * 2) : 0;
  o->f_index = K ? take(rows * k * 4) : 0;
  o->f_logit = K ? take(rows * k * 4) : 0;
  o->f_entry_z = K ? take(rows * k * 4) : 0;
  o->f_info = K ? take(rows * 4) : 0;
  o->f_total = off;
  off = align_up(sizeof(ObjHeader), 256);
  o->s_rows = take((size_t)S * sizeof(ObjRow));
  o->s_rows2 = K ? take((size_t)S * sizeof(ObjRow2)) : 0;
  o->s_index = K ? take((size_t)S * k * 4) : 0;
  o->s_at = K ? take((size_t)S * k * 4) : 0;
  o->s_total = off;
  return MST_OK;
}

struct ObjCall {       // a forward call's arguments, of either objective
  const void *H, *W;
  const int32_t* labels;
  const float* weights;
  const int32_t* index;
  const void* logits;
  int32_t logits_bf16;
  const float* teacher_lse;
  int32_t ignore_index;
  float softcap, label_coef, teacher_coef, temperature, z_coef;
  int64_t divisor;
  void* workspace;
  size_t workspace_bytes;
  void* saved;
  size_t saved_bytes;
  float *loss, *nll, *kd, *lse;
  int64_t* n_valid;
  void* stream;
};

template <bool kAll>
auto finalize_kernel_of(int K) {
  return K == 0 ? k_obj_finalize<kAll, 0> : K <= 16 ? k_obj_finalize<kAll, 1> : K <= 32 ? k_obj_finalize<kAll, 2>
       : K <= 64 ? k_obj_finalize<kAll, 4> : K <= 128 ? k_obj_finalize<kAll, 8> : k_obj_finalize<kAll, 16>;
}
auto finalize_kernel(bool all, int K) { return all ? finalize_kernel_of<true>(K) : finalize_kernel_of<false>(K); }

mst_status obj_forward(const ObjPlan& o, const ObjCall& c) {
  const Plan& p = o.p;
  const size_t rows = (size_t)p.S, k = (size_t)o.K;
  if (!c.H || !c.W || !c.loss || (o.K ? !c.index || !c.logits : !c.labels)) return MST_ERR_NULL_POINTER;
  const bool good_cap = c.softcap == 0.f || (c.softcap >= 1e-3f && c.softcap <= 1e6f);
  if (!good_cap || !std::isfinite(c.label_coef) || !std::isfinite(c.teacher_coef) || !std::isfinite(c.z_coef) ||
      !(c.temperature >= 0.01f && c.temperature <= 100.f) || c.divisor < 0 || (!c.labels && (c.label_coef != 0.f || c.nll)))
    return MST_ERR_BAD_ARGUMENT;
  if (!c.workspace || c.workspace_bytes < o.f_total || (c.saved && c.saved_bytes < o.s_total)) return MST_ERR_WORKSPACE;
  if (misaligned(c.H, 16) || misaligned(c.W, 16) || misaligned(c.workspace, 256) || misaligned(c.saved, 256) || misaligned(c.labels, 4) ||
      misaligned(c.weights, 4) || misaligned(c.index, 4) || misaligned(c.logits, c.logits_bf16 ? 2 : 4) || misaligned(c.teacher_lse, 4) ||
      misaligned(c.loss, 4) || misaligned(c.nll, 4) || misaligned(c.kd, 4) || misaligned(c.lse, 4) || misaligned(c.n_valid, 8))
    return MST_ERR_ALIGNMENT;
  Ranges ranges;
  ranges.add(c.H, rows * p.d * 2, false);
  ranges.add(c.W, (size_t)p.V * p.d * 2, false);
  ranges.add(c.labels, rows * 4, false);
  ranges.add(c.weights, rows * 4, false);
  ranges.add(c.index, rows * k * 4, false);
  ranges.add(c.logits, rows * k * (c.logits_bf16 ? 2 : 4), false);
  ranges.add(c.teacher_lse, rows * 4, false);
  ranges.add(c.workspace, o.f_total, true);
  ranges.add(c.saved, o.s_total, true);
  ranges.add(c.loss, 4, true);
  ranges.add(c.nll, rows * 4, true);
  ranges.add(c.kd, rows * 4, true);
  ranges.add(c.lse, rows * 4, true);
  ranges.add(c.n_valid, 8, true);
  if (!ranges.apart()) return MST_ERR_BAD_ARGUMENT;
  mst_status s = prepare_device();
  if (s != MST_OK) return s;

  hipStream_t st = reinterpret_cast<hipStream_t>(c.stream);
  char* const ws = static_cast<char*>(c.workspace);
  char* const saved = static_cast<char*>(c.saved);
  const size_t stride = (size_t)p.fwd_group_rows;
  // both log-sum-exps, at 1 / T for the teacher and at 1 for the labels, only where they differ and the second is asked for
  const bool two = o.K && c.labels && (c.label_coef != 0.f || c.nll) && c.temperature != 1.f;
  const float exponent = (float)(1.4426950408889634 / (double)c.temperature);
  ObjTile e = {};
  e.part = reinterpret_cast<float2*>(ws + (o.few ? o.f_part_few : p.f_part));
  e.part_label = two ? reinterpret_cast<float*>(ws + o.f_part_label) : nullptr;
  e.part_stride = stride;
  e.tgt = reinterpret_cast<float*>(ws + p.f_tgt);
  e.K = o.K;
  e.cap = c.softcap;
  e.exponent = exponent;
  e.exponent_label = kLog2e;
  int* const index = reinterpret_cast<int*>(ws + o.f_index);
  float* const logit = reinterpret_cast<float*>(ws + o.f_logit);
  int* const info = reinterpret_cast<int*>(ws + o.f_info);
  unsigned short* const starts = reinterpret_cast<unsigned short*>(ws + o.f_starts);
  const bool sorted = o.K && !o.few && forward_tile_rows(p) > 32;
  if (o.K) {
    e.starts = sorted ? starts : nullptr;
    e.index = index;
    e.entry_z = reinterpret_cast<float*>(ws + o.f_entry_z);
    e.info = info;
  }
  ObjFinal f = {};
  f.part = e.part; f.part_label = e.part_label; f.part_stride = stride;
  f.n_vt = o.n_vt; f.V = (int)p.V; f.K = o.K;
  f.tgt = e.tgt; f.ignore_index = c.ignore_index;
  f.index = index; f.logit = sorted ? logit : nullptr; f.logit_bf16 = c.logits_bf16; f.entry_z = e.entry_z; f.info = info;
  f.cap = c.softcap; f.exponent = exponent; f.exponent_label = kLog2e; f.inv_t_64 = 1.0 / (double)c.temperature; f.inv_t = (float)f.inv_t_64;
  f.label_coef = c.label_coef; f.teacher_coef = c.teacher_coef; f.z_coef = c.z_coef; f.temperature = c.temperature;
  // The logits' gradient is rounded to bf16, entry by entry, which errors of either sign survive and a common factor of all rows does not
  // (a label's gradient is its coefficient times nearly -1: 0.3 is 0.3008 in bf16, a label's part of dH and dW 0.26 % too large).  The part of
  // the labels' coefficient, or the teacher's alone, that has to be rounded, from 1 to 2, therefore goes into the divisor.
  auto mantissa = [](double x) { int e; return x == 0.0 ? 1.0 : 2.0 * std::frexp(std::fabs(x), &e); };
  const double slope = (double)c.teacher_coef * (double)c.temperature;
  const double unit = c.labels && c.label_coef != 0.f ? mantissa(c.label_coef) : mantissa(slope);
  f.label_slope = (float)((double)c.label_coef / unit); f.teacher_slope = (float)(slope / unit); f.z_slope = (float)((double)c.z_coef / unit);
  float2* const row_loss = reinterpret_cast<float2*>(ws + o.f_row_loss);

  ObjLoss l = {};
  l.divisor = c.divisor;
  l.unit = unit;
  l.head.cap = c.softcap;
  l.head.exponent = exponent;
  l.head.exponent_label = kLog2e;
  l.head.two = two;
  l.saved = reinterpret_cast<ObjHeader*>(saved);
  l.loss = c.loss;
  l.n_valid = reinterpret_cast<long long*>(c.n_valid);
  const bool one_group = p.S <= kObjRows && p.S <= p.fwd_group_rows;       // the call's rows are one workgroup of k_obj_finalize
  const bool lone = !one_group && one_finalizes(o);
  const bool one = lone || one_group;                                      // the loss is formed with the rows' losses
  auto logits_from = [&](int64_t g0) -> const void* { return static_cast<const char*>(c.logits) + (size_t)g0 * k * (c.logits_bf16 ? 2 : 4); };
  auto tile_of = [&](int64_t g0) {
    ObjTile of = e;
    of.labels_c = c.labels ? c.labels + g0 : nullptr;
    if (o.K) of.index_in_c = c.index + (size_t)g0 * k;
    return of;
  };
  auto before = [&](int64_t g0, int g_rows) {
    if (!sorted) return;
    Scope sc(st, MST_K_LABEL_SCAN);
    const auto kernel = o.K <= 64 ? k_entries<1> : o.K <= 128 ? k_entries<2> : k_entries<4>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((g_rows + kEntryRows - 1) / kEntryRows)), dim3(64 * kEntryRows), 0, st,
                       c.index + (size_t)g0 * k, logits_from(g0), c.logits_bf16, g_rows, o.K, (int)p.V, p.n_vt, index, logit, info, starts, stride);
  };
  auto after = [&](int64_t g0, int g_rows) {
    ObjFinal of = f;
    of.rows = g_rows;
    if (o.K) of.logit_in_c = logits_from(g0);
    of.labels_c = c.labels ? c.labels + g0 : nullptr;
    of.weights_c = c.weights ? c.weights + g0 : nullptr;
    of.teacher_lse_c = c.teacher_lse ? c.teacher_lse + g0 : nullptr;
    of.nll_c = c.nll ? c.nll + g0 : nullptr;
    of.kd_c = c.kd ? c.kd + g0 : nullptr;
    of.lse_c = c.lse ? c.lse + g0 : nullptr;
    of.row_loss_c = row_loss + g0;
    if (saved) {
      of.rows_c = reinterpret_cast<ObjRow*>(saved + o.s_rows) + g0;
      if (o.K) {
        of.rows2_c = reinterpret_cast<ObjRow2*>(saved + o.s_rows2) + g0;
        of.saved_index_c = reinterpret_cast<int*>(saved + o.s_index) + (size_t)g0 * k;
        of.saved_at_c = reinterpret_cast<float*>(saved + o.s_at) + (size_t)g0 * k;
      }
    }
    Scope sc(st, MST_K_LSE_FINALIZE);
    if (lone) {
      hipLaunchKernelGGL(k_obj_finalize_one, dim3(1), dim3(1024), 0, st, of, l, finalize_row_bits(p.S, o.n_vt));
      return;
    }
    hipLaunchKernelGGL(finalize_kernel(one, o.K), dim3((unsigned)((g_rows + kObjRows - 1) / kObjRows)), dim3(kObjRows * kObjGroups), 0, st, of, l);
  };
  const __bf16 *const H = static_cast<const __bf16*>(c.H), *const W = static_cast<const __bf16*>(c.W);
  if (o.few) {
    {
      Scope sc(st, MST_K_FWD_GEMM_LSE);
      hipLaunchKernelGGL((k_fwd_gemm_lse_small<TileFew, ObjEpilogue<kObjAny>>), dim3(even_grid(o.n_vt, few_row_tiles(p))), dim3(TileFew::kThreads),
                         TileFew::kLds, st, H, W, (int)p.S, (int)p.d, (int)p.V, few_row_tiles(p), o.n_vt, ObjEpilogue<kObjAny>(tile_of(0)));
    }
    after(0, (int)p.S);
  } else {
    auto run = [&](auto what) {
      return run_forward_groups(p, H, W, st, reinterpret_cast<Control*>(ws),
                                [&](int64_t g0) { return ObjEpilogue<decltype(what)::value>(tile_of(g0)); }, before, after);
    };
    s = o.K ? run(std::integral_constant<int, kObjAny>())
            : c.softcap > 0.f ? run(std::integral_constant<int, kObjCap>()) : run(std::integral_constant<int, 0>());
    if (s != MST_OK) return s;
  }
  if (!one) {
    Scope sc(st, MST_K_LOSS_REDUCE);
    hipLaunchKernelGGL(k_obj_loss, dim3(1), dim3(1024), 0, st, row_loss, (long long)p.S, l);
  }
  return check_launch();
}

mst_status obj_backward(const ObjPlan& o, const void* H, const void* W, float grad_loss, const void* saved_in, size_t saved_bytes,
                        void* workspace, size_t workspace_bytes, void* dH, float* dW, void* stream) {
  const Plan& p = o.p;
  if (!H || !W || !saved_in || !dH || !dW) return MST_ERR_NULL_POINTER;
  if (!workspace || workspace_bytes < p.b_total || saved_bytes < o.s_total) return MST_ERR_WORKSPACE;
  if (misaligned(H, 16) || misaligned(W, 16) || misaligned(dH, 16) || misaligned(dW, 16) || misaligned(workspace, 256) || misaligned(saved_in, 256))
    return MST_ERR_ALIGNMENT;
  Ranges ranges;
  ranges.add(H, (size_t)p.S * p.d * 2, false);
  ranges.add(W, (size_t)p.V * p.d * 2, false);
  ranges.add(saved_in, o.s_total, false);
  ranges.add(workspace, p.b_total, true);
  ranges.add(dH, (size_t)p.S * p.d * 2, true);
  ranges.add(dW, (size_t)p.V * p.d * 4, true);
  if (!ranges.apart()) return MST_ERR_BAD_ARGUMENT;
  mst_status s = prepare_device();
  if (s != MST_OK) return s;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const char* const saved = static_cast<const char*>(saved_in);
  const ObjHeader* const head = reinterpret_cast<const ObjHeader*>(saved);
  const ObjRow* const rows = reinterpret_cast<const ObjRow*>(saved + o.s_rows);
  const ObjRow2* const rows2 = o.K ? reinterpret_cast<const ObjRow2*>(saved + o.s_rows2) : nullptr;
  const int* const index = reinterpret_cast<const int*>(saved + o.s_index);
  const float* const at = reinterpret_cast<const float*>(saved + o.s_at);
  return run_backward_orders(
      p, static_cast<const __bf16*>(H), static_cast<const __bf16*>(W), &head->n_divisor, grad_loss, static_cast<char*>(workspace),
      static_cast<__bf16*>(dH), dW, st,
      [&](int64_t r0) {
        const bool patch = o.K && o.K <= kPatchEntries;
        return ObjGrad{head, rows + r0, rows2 ? rows2 + r0 : nullptr, index + (size_t)r0 * o.K, at + (size_t)r0 * o.K, patch ? o.K : 0};
      },
      [&](int64_t r0, int n_rows, int64_t v_base, int Vw, __bf16* G, int ldg, bool small) {
        if (!o.K || (small && o.K <= kPatchEntries)) return;
        const size_t from = (size_t)r0 * o.K;
        const long long n = (long long)n_rows * o.K;
        Scope sc(st, MST_K_BWD_DH_REDUCE);
        hipLaunchKernelGGL(k_obj_entries, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, index + from, at + from, n, o.K, (int)v_base, Vw, G,
                           ldg);
      });
}

}  // namespace

extern "C" {

mst_status mst_objective_bytes(int64_t S, int64_t d, int64_t V, int32_t M, int32_t K, size_t* fwd_bytes, size_t* bwd_bytes, size_t* saved_bytes) {
  ObjPlan o;
  const mst_status s = make_obj_plan(S, d, V, M, K, &o);
  if (s != MST_OK) return s;
  if (fwd_bytes) *fwd_bytes = o.f_total;
  if (bwd_bytes) *bwd_bytes = o.p.b_total;
  if (saved_bytes) *saved_bytes = o.s_total;
  return MST_OK;
}

mst_status mst_lmhead_wce_fwd(const void* H, const void* W, const int32_t* labels, const float* weights, int64_t S, int64_t d, int64_t V,
                              int32_t ignore_index, int32_t M, float softcap, float z_coef, int64_t divisor, void* workspace,
                              size_t workspace_bytes, void* saved, size_t saved_bytes, float* loss, float* nll, float* lse, int64_t* n_valid,
                              void* stream) {
  ObjPlan o;
  const mst_status s = make_obj_plan(S, d, V, M, 0, &o);
  if (s != MST_OK) return s;
  return obj_forward(o, {H, W, labels, weights, nullptr, nullptr, 0, nullptr, ignore_index, softcap, 1.f, 0.f, 1.f, z_coef, divisor, workspace,
                         workspace_bytes, saved, saved_bytes, loss, nll, nullptr, lse, n_valid, stream});
}

mst_status mst_lmhead_wce_bwd(const void* H, const void* W, int64_t S, int64_t d, int64_t V, int32_t M, float grad_loss, const void* saved,
                              size_t saved_bytes, void* workspace, size_t workspace_bytes, void* dH, float* dW, void* stream) {
  ObjPlan o;
  const mst_status s = make_obj_plan(S, d, V, M, 0, &o, t_bwd_schedule, true);
  if (s != MST_OK) return s;
  return obj_backward(o, H, W, grad_loss, saved, saved_bytes, workspace, workspace_bytes, dH, dW, stream);
}

mst_status mst_lmhead_distill_fwd(const void* H, const void* W, const int32_t* labels, const float* weights, const int32_t* teacher_index,
                                  const void* teacher_logits, int32_t teacher_type, const float* teacher_lse, int64_t S, int64_t d, int64_t V,
                                  int32_t K, int32_t ignore_index, int32_t M, float softcap, float label_coef, float teacher_coef,
                                  float temperature, int64_t divisor, void* workspace, size_t workspace_bytes, void* saved, size_t saved_bytes,
                                  float* loss, float* nll, float* kd, int64_t* n_valid, void* stream) {
  if (K < 1) return MST_ERR_BAD_SHAPE;
  ObjPlan o;
  const mst_status s = make_obj_plan(S, d, V, M, K, &o);
  if (s != MST_OK) return s;
  if (teacher_type != 0 && teacher_type != 1) return MST_ERR_BAD_ARGUMENT;
  return obj_forward(o, {H, W, labels, weights, teacher_index, teacher_logits, teacher_type == 0, teacher_lse, ignore_index, softcap, label_coef,
                         teacher_coef, temperature, 0.f, divisor, workspace, workspace_bytes, saved, saved_bytes, loss, nll, kd, nullptr, n_valid,
                         stream});
}

mst_status mst_lmhead_distill_bwd(const void* H, const void* W, int64_t S, int64_t d, int64_t V, int32_t K, int32_t M, float grad_loss,
                                  const void* saved, size_t saved_bytes, void* workspace, size_t workspace_bytes, void* dH, float* dW,
                                  void* stream) {
  if (K < 1) return MST_ERR_BAD_SHAPE;
  ObjPlan o;
  const mst_status s = make_obj_plan(S, d, V, M, K, &o, t_bwd_schedule, true);
  if (s != MST_OK) return s;
  return obj_backward(o, H, W, grad_loss, saved, saved_bytes, workspace, workspace_bytes, dH, dW, stream);
}

}  // extern "C"
