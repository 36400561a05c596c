// Host side of the norm, residual and checkpoint calls: argument validation, workspace carving, launches.
#include "../../include/mst_norm.h"
#include "host_util.hpp"
#include "norm_launch.hpp"

#include <algorithm>
#include <cmath>

namespace {

using namespace mst;
using namespace mst_norm;
using mst_host::misaligned;

constexpr int kNumCu = 256;

mst_status check_shape(int64_t S, int64_t d) {
  if (S < 1 || S >= (int64_t(1) << 30) || d < 8 || d % 8 != 0 || d > MST_NORM_MAX_D || S * d > (int64_t(1) << 36)) return MST_ERR_BAD_SHAPE;
  return MST_OK;
}

// The tensors of a call, to be checked in one go.
struct Operands {
  struct Range { uintptr_t at; size_t bytes; int entry; bool out, whole; };
  Range r[24];
  int n = 0;
  bool aligned = true;
  // entry: bytes of an entry; whole: one entry for each row and column
  void add(const void* p, int64_t entries, int entry, bool out, bool whole, size_t alignment = 16) {
    if (!p) return;
    if (misaligned(p, alignment)) aligned = false;
    r[n++] = {reinterpret_cast<uintptr_t>(p), (size_t)entries * entry, entry, out, whole};
  }
  mst_status check() const {
    if (!aligned) return MST_ERR_ALIGNMENT;
    for (int i = 0; i < n; ++i)
      for (int j = 0; j < i; ++j) {
        const Range &a = r[i], &b = r[j];
        if (!(a.out || b.out) || a.at >= b.at + b.bytes || b.at >= a.at + a.bytes) continue;
        // a lane reads its entries of an input before it writes the same ones of an output
        if (a.out == b.out || !a.whole || !b.whole || a.at != b.at || a.entry != b.entry) return MST_ERR_BAD_ARGUMENT;
      }
    return MST_OK;
  }
};

int type_bytes(int32_t type) { return type == MST_TYPE_FP32 ? 4 : 2; }
bool good_type(int32_t type) { return type == MST_TYPE_BF16 || type == MST_TYPE_FP32; }

// Gate and scale; rows of the gate in *rows (0 without one).
mst_status check_gate(const void* gate, int64_t gate_rows, float scale, int64_t S, int64_t* rows) {
  if (!std::isfinite(scale) || (gate ? gate_rows < 1 : gate_rows != 0)) return MST_ERR_BAD_ARGUMENT;
  *rows = gate ? (S + std::min(gate_rows, S) - 1) / std::min(gate_rows, S) : 0;
  return MST_OK;
}

// Up to so many rows of each team that a workgroup has room for are left to one workgroup: no sums to join, one launch.  2 rows of
// 4096, norm: 5.4 us, in workgroups of their own 6.6; 4 rows of a team 10.8.
constexpr int kAloneRows = 2;

// How the backward calls deal out the rows (k_norm_bwd).  gate_rows: 0 without a gate; pre: with the norm before a block.
//   Workgroups: a compute unit is given one or more whose lanes have 512 times eight columns together (lanes behind a row's end not counted); in the
//   residual's backward alone, which loads half as much, as many as fit 1024 lanes (all counted).  That is about 40 KB of loads under way.  More of them
//   pass through more rows at a time and are slower for it: 32768 x 4096, us, with one and with two workgroups of 512 lanes: norm 160, 162 (155, 180
//   with two rows ahead), both norms 243, 263, residual 138, 118.
//   Rows of the gate: whole ones to a team where there are as many as teams (half as many for the residual's backward), or where a row of the gate
//   has fewer rows than a workgroup has teams; else `share` workgroups each.  Whole against shared, us, 8192 x 1024, both
//   norms, 1 row of the gate for 8 rows: 27, 29, for 16: 37, 23; residual: for 8 18, 20, for 16 24, 17; 32768 x 256, both
//   norms, for 8 28, 60.
struct BwdPlan {
  RowPlan row;
  bool whole;                            // teams take whole rows of the gate
  int64_t gates, share, groups;          // rows of the gate (1 without); workgroups of each; workgroups
  int rows;                              // that a team takes in turn
  BwdPlan(int64_t S, int64_t d, int64_t gate_rows, bool pre) : row(d) {
    const int64_t L = gate_rows ? std::min(gate_rows, S) : S;
    const int lanes = (int)(row.teams * d / 8);                           // of a workgroup, that have columns
    const int64_t most = kNumCu * std::max(1, pre ? (512 + lanes / 2) / lanes : 1024 / row.threads());
    gates = (S + L - 1) / L;
    whole = gates > 1 && ((pre ? 1 : 2) * gates >= most * row.teams || L < row.teams) && L * row.teams * d < (int64_t(1) << 29);
    if (whole) {
      groups = std::min(most, (gates + row.teams - 1) / row.teams);
      share = 0;
      rows = (int)((gates + groups * row.teams - 1) / (groups * row.teams) * L);
      return;
    }
    const int most_teams = 1024 / (row.team.lanes * row.team.waves);
    if (gates == 1 && S <= kAloneRows * most_teams) {
      row.teams = most_teams;
      rows = (int)((S + most_teams - 1) / most_teams);
      share = groups = 1;
      return;
    }
    const int64_t wanted = (most + gates - 1) / gates;
    rows = (int)((L + wanted * row.teams - 1) / (wanted * row.teams));
    share = (L + (int64_t)rows * row.teams - 1) / ((int64_t)rows * row.teams);
    groups = gates * share;
  }
};

size_t workspace_bytes(const BwdPlan& p, int64_t d) {      // dw_pre and dw_post by workgroup
  return mst_host::align_up(p.groups > 1 ? 2 * (size_t)p.groups * d * 4 : 1, 256);
}

template <class T, bool kPre, bool kRes, bool kWhole, bool kCkptX, bool kCkptO, int kPolicy>
mst_status launch_bwd(NormBwd a, const BwdPlan& p, void* workspace, hipStream_t st) {
  a.rows = p.rows;
  a.share = (int)p.share;
  a.team = p.row.team;
  a.part_pre = static_cast<float*>(workspace);
  a.part_post = a.part_pre + (size_t)p.groups * a.d;
  const dim3 grid((unsigned)p.groups), block(p.row.threads());
  const size_t lds = p.row.teams > 1 ? (size_t)p.row.teams * a.d * 4 : 0;      // 16 KB of 512 lanes, 32 of a lone workgroup
  if (p.row.chunks == 1)
    hipLaunchKernelGGL((k_norm_bwd<T, kPre, kRes, kWhole, kCkptX, kCkptO, kPolicy, 1>), grid, block, lds, st, a);
  else
    hipLaunchKernelGGL((k_norm_bwd<T, kPre, kRes, kWhole, kCkptX, kCkptO, kPolicy, 2>), grid, block, lds, st, a);
  if (p.groups > 1 && (a.dw_pre || a.dw_post || (a.dgate && !kWhole))) {      // teams of whole rows of the gate have written dgate
    int slices = 1;                                       // of the sums of a row of the gate
    while (slices < kReduceSlices && slices < p.share) slices *= 2;
    const int64_t per_block = kReduceSlices / slices, gates = a.dgate && !kWhole && p.gates > 1 ? (p.gates + per_block - 1) / per_block : 0;
    hipLaunchKernelGGL(k_norm_reduce, dim3((a.d + kReduceCols - 1) / kReduceCols, (unsigned)(2 + gates)), dim3(kReduceThreads), 0, st, a,
                       (int)p.groups, (int)kWhole, slices);
  }
  return launched();
}

template <class T, bool kPre, bool kRes>
mst_status dispatch_bwd(NormBwd a, int64_t gate_rows, void* workspace, hipStream_t st) {
  constexpr bool kX = kPre, kO = kRes;             // where there can be a checkpoint
  const BwdPlan p(a.S, a.d, gate_rows, kPre);
  a.gate_rows = (int)(gate_rows ? std::min<int64_t>(gate_rows, a.S) : a.S);
  a.gates = (int)p.gates;
  auto go = [&](auto w, auto stream) {
    constexpr bool kWhole = kRes && decltype(w)::value;
    constexpr int kPolicy = decltype(stream)::value ? kNonTemporalAccess : 0;
    if (a.codes_x && a.codes_o) return launch_bwd<T, kPre, kRes, kWhole, kX, kO, kPolicy>(a, p, workspace, st);
    if (a.codes_x) return launch_bwd<T, kPre, kRes, kWhole, kX, false, kPolicy>(a, p, workspace, st);
    if (a.codes_o) return launch_bwd<T, kPre, kRes, kWhole, false, kO, kPolicy>(a, p, workspace, st);
    return launch_bwd<T, kPre, kRes, kWhole, false, false, kPolicy>(a, p, workspace, st);
  };
  const int64_t n = (int64_t)a.S * a.d, t = sizeof(T);
  const bool stream = n * ((kPre ? 2 + 2 * t + (a.codes_x ? 1 : t) : t) + (kRes ? 3 : 0)) > kCacheBytes;
  if (p.whole) return stream ? go(std::true_type(), std::true_type()) : go(std::true_type(), std::false_type());
  return stream ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
}
template <bool kPre, bool kRes>
mst_status dispatch_bwd(const NormBwd& a, int32_t type, int64_t gate_rows, void* workspace, hipStream_t st) {
  return type == MST_TYPE_FP32 ? dispatch_bwd<float, kPre, kRes>(a, gate_rows, workspace, st)
                               : dispatch_bwd<__bf16, kPre, kRes>(a, gate_rows, workspace, st);
}

// The rows are dealt out to the workgroups of a whole chip (BwdPlan): a partitioned device is refused.
mst_host::PerDeviceOnce g_shape_once;
mst_status check_device() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return MST_ERR_NO_DEVICE;
  if (g_shape_once.run(dev, [dev] { return mst_host::has_compute_units(dev, kNumCu); })) return MST_OK;
  (void)hipGetLastError();
  return MST_ERR_NO_DEVICE;
}

bool both_or_neither(const void* a, const void* b) { return !a == !b; }
const __bf16* bf(const void* p) { return static_cast<const __bf16*>(p); }
hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

const char* mst_norm_version(void) { return "mst-norm 0.1 (gfx950)"; }

mst_status mst_norm_workspace_bytes(int64_t S, int64_t d, int64_t gate_rows, size_t* bytes) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (gate_rows < 0) return MST_ERR_BAD_ARGUMENT;
  if (!bytes) return MST_ERR_NULL_POINTER;
  *bytes = std::max(workspace_bytes(BwdPlan(S, d, gate_rows, false), d), workspace_bytes(BwdPlan(S, d, gate_rows, true), d));
  return MST_OK;
}

mst_status mst_norm_bwd_info(int64_t S, int64_t d, int64_t gate_rows, int32_t prenorm, int64_t* info) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (gate_rows < 0) return MST_ERR_BAD_ARGUMENT;
  if (!info) return MST_ERR_NULL_POINTER;
  const BwdPlan p(S, d, gate_rows, prenorm != 0);
  info[0] = p.row.threads();
  info[1] = p.row.teams;
  info[2] = p.rows;
  info[3] = p.groups;
  info[4] = p.whole;
  return MST_OK;
}

mst_status mst_ckpt_pack(const void* X, int32_t type, int64_t S, int64_t d, int8_t* codes, uint8_t* exps, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (!X || !codes || !exps) return MST_ERR_NULL_POINTER;
  if (!good_type(type)) return MST_ERR_BAD_ARGUMENT;
  Operands ops;
  ops.add(X, S * d, type_bytes(type), false, true);
  ops.add(codes, S * d, 1, true, true);
  ops.add(exps, S * blocks_of_row(d), 1, true, false, 1);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  if (type == MST_TYPE_FP32) launch_pack(static_cast<const float*>(X), S, d, codes, exps, as_stream(stream));
  else launch_pack(bf(X), S, d, codes, exps, as_stream(stream));
  return launched();
}

mst_status mst_ckpt_unpack(const int8_t* codes, const uint8_t* exps, int64_t S, int64_t d, void* X, int32_t type, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (!X || !codes || !exps) return MST_ERR_NULL_POINTER;
  if (!good_type(type)) return MST_ERR_BAD_ARGUMENT;
  Operands ops;
  ops.add(X, S * d, type_bytes(type), true, true);
  ops.add(codes, S * d, 1, false, true);
  ops.add(exps, S * blocks_of_row(d), 1, false, false, 1);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  if (type == MST_TYPE_FP32) launch_unpack(codes, exps, S, d, static_cast<float*>(X), as_stream(stream));
  else launch_unpack(codes, exps, S, d, static_cast<__bf16*>(X), as_stream(stream));
  return launched();
}

mst_status mst_prenorm_fwd(const void* X, int32_t stream_type, const void* w_pre, float w_offset, float eps,
                           int64_t S, int64_t d, void* H, int8_t* codes, uint8_t* exps, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (!X || !H) return MST_ERR_NULL_POINTER;
  if (!good_type(stream_type) || !good_norm(eps, w_offset) || !both_or_neither(codes, exps)) return MST_ERR_BAD_ARGUMENT;
  Operands ops;
  ops.add(X, S * d, type_bytes(stream_type), false, true);
  ops.add(w_pre, d, 2, false, false);
  ops.add(H, S * d, 2, true, true);
  ops.add(codes, S * d, 1, true, true);
  ops.add(exps, S * blocks_of_row(d), 1, true, false, 1);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  NormFwd a = {};
  a.X = X; a.w_pre = bf(w_pre); a.H = static_cast<__bf16*>(H);
  a.codes_y = codes; a.exps_y = exps;
  a.offset = w_offset; a.eps = eps; a.inv_d = 1.f / (float)d;
  a.S = (int)S; a.d = (int)d; a.gate_rows = (int)S; a.gates = 1;
  return stream_type == MST_TYPE_FP32 ? launch_fwd<float, false, true, false>(a, as_stream(stream))
                                      : launch_fwd<__bf16, false, true, false>(a, as_stream(stream));
}

mst_status mst_prenorm_rebuild(const int8_t* codes, const uint8_t* exps, const void* w_pre, float w_offset, float eps,
                               int64_t S, int64_t d, void* H, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (!codes || !exps || !H) return MST_ERR_NULL_POINTER;
  if (!good_norm(eps, w_offset)) return MST_ERR_BAD_ARGUMENT;
  Operands ops;
  ops.add(codes, S * d, 1, false, true);
  ops.add(exps, S * blocks_of_row(d), 1, false, false, 1);
  ops.add(w_pre, d, 2, false, false);
  ops.add(H, S * d, 2, true, true);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  NormFwd a = {};
  a.codes_x = codes; a.exps_x = exps; a.w_pre = bf(w_pre); a.H = static_cast<__bf16*>(H);
  a.offset = w_offset; a.eps = eps; a.inv_d = 1.f / (float)d;
  a.S = (int)S; a.d = (int)d; a.gate_rows = (int)S; a.gates = 1;
  return launch_fwd<__bf16, false, true, true>(a, as_stream(stream));
}

mst_status mst_prenorm_bwd(const void* dH, const void* X, const int8_t* codes, const uint8_t* exps, const void* dres,
                           int32_t stream_type, const void* w_pre, float w_offset, float eps, int64_t S, int64_t d,
                           void* workspace, size_t workspace_size, void* dX, float* dw_pre, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (!dH || !dX || (!X && !codes && !exps)) return MST_ERR_NULL_POINTER;
  if (!good_type(stream_type) || !good_norm(eps, w_offset) || !both_or_neither(codes, exps) || (X && codes) || (dw_pre && !w_pre))
    return MST_ERR_BAD_ARGUMENT;
  if (w_pre && !dw_pre) return MST_ERR_NULL_POINTER;
  const size_t need = workspace_bytes(BwdPlan(S, d, 0, true), d);
  if (!workspace || workspace_size < need) return MST_ERR_WORKSPACE;
  Operands ops;
  ops.add(dH, S * d, 2, false, true);
  ops.add(X, S * d, type_bytes(stream_type), false, true);
  ops.add(codes, S * d, 1, false, true);
  ops.add(exps, S * blocks_of_row(d), 1, false, false, 1);
  ops.add(dres, S * d, type_bytes(stream_type), false, true);
  ops.add(w_pre, d, 2, false, false);
  ops.add(workspace, (int64_t)need, 1, true, false, 256);
  ops.add(dX, S * d, type_bytes(stream_type), true, true);
  ops.add(dw_pre, d, 4, true, false);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  NormBwd a = {};
  a.dH = bf(dH); a.dres = dres; a.X = X; a.codes_x = codes; a.exps_x = exps; a.w_pre = bf(w_pre);
  a.dX = dX; a.dw_pre = dw_pre;
  a.offset = w_offset; a.eps = eps; a.scale = 1.f; a.inv_d = 1.f / (float)d;
  a.S = (int)S; a.d = (int)d;
  return dispatch_bwd<true, false>(a, stream_type, 0, workspace, as_stream(stream));
}

mst_status mst_residual_fwd(const void* O, const void* X, int32_t stream_type, int32_t normalize, const void* w_post,
                            float w_offset, float eps, const void* gate, int64_t gate_rows, float scale,
                            int64_t S, int64_t d, void* Y, int8_t* codes, uint8_t* exps, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (!O || !X || !Y) return MST_ERR_NULL_POINTER;
  int64_t gate_groups = 0;
  if ((s = check_gate(gate, gate_rows, scale, S, &gate_groups)) != MST_OK) return s;
  if (!good_type(stream_type) || !good_norm(eps, w_offset) || !both_or_neither(codes, exps) || (w_post && !normalize)) return MST_ERR_BAD_ARGUMENT;
  Operands ops;
  ops.add(O, S * d, 2, false, true);
  ops.add(X, S * d, type_bytes(stream_type), false, true);
  ops.add(w_post, d, 2, false, false);
  ops.add(gate, gate_groups * d, 2, false, false);
  ops.add(Y, S * d, type_bytes(stream_type), true, true);
  ops.add(codes, S * d, 1, true, true);
  ops.add(exps, S * blocks_of_row(d), 1, true, false, 1);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  NormFwd a = {};
  a.X = X; a.O = bf(O); a.w_post = bf(w_post); a.gate = bf(gate); a.Y = Y;
  a.codes_o = codes; a.exps_o = exps;
  a.offset = w_offset; a.eps = eps; a.scale = scale; a.inv_d = 1.f / (float)d;
  a.S = (int)S; a.d = (int)d; a.normalize = normalize != 0;
  a.gate_rows = (int)(gate ? std::min(gate_rows, S) : S);
  a.gates = (int)std::max<int64_t>(gate_groups, 1);
  return stream_type == MST_TYPE_FP32 ? launch_fwd<float, true, false, false>(a, as_stream(stream))
                                      : launch_fwd<__bf16, true, false, false>(a, as_stream(stream));
}

mst_status mst_residual_bwd(const void* dY, int32_t stream_type, const void* O, const int8_t* codes, const uint8_t* exps,
                            int32_t normalize, const void* w_post, float w_offset, float eps,
                            const void* gate, int64_t gate_rows, float scale, int64_t S, int64_t d,
                            void* workspace, size_t workspace_size, void* dO, float* dw_post, float* dgate, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  int64_t gate_groups = 0;
  if ((s = check_gate(gate, gate_rows, scale, S, &gate_groups)) != MST_OK) return s;
  if (!dY || !dO) return MST_ERR_NULL_POINTER;
  if (!good_type(stream_type) || !good_norm(eps, w_offset) || !both_or_neither(codes, exps) || (O && codes) || (w_post && !normalize) ||
      (dw_post && !w_post) || (dgate && !gate))
    return MST_ERR_BAD_ARGUMENT;
  if ((w_post && !dw_post) || (gate && !dgate) || ((normalize || gate) && !O && !codes)) return MST_ERR_NULL_POINTER;
  const size_t need = workspace_bytes(BwdPlan(S, d, gate_rows, false), d);
  if (!workspace || workspace_size < need) return MST_ERR_WORKSPACE;
  if (!normalize && !gate) O = nullptr, codes = nullptr, exps = nullptr;
  Operands ops;
  ops.add(dY, S * d, type_bytes(stream_type), false, true);
  ops.add(O, S * d, 2, false, true);
  ops.add(codes, S * d, 1, false, true);
  ops.add(exps, S * blocks_of_row(d), 1, false, false, 1);
  ops.add(w_post, d, 2, false, false);
  ops.add(gate, gate_groups * d, 2, false, false);
  ops.add(workspace, (int64_t)need, 1, true, false, 256);
  ops.add(dO, S * d, 2, true, true);
  ops.add(dw_post, d, 4, true, false);
  ops.add(dgate, gate_groups * d, 4, true, false);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  NormBwd a = {};
  a.dY = dY; a.O = bf(O); a.codes_o = codes; a.exps_o = exps; a.w_post = bf(w_post); a.gate = bf(gate);
  a.dO = static_cast<__bf16*>(dO); a.dw_post = dw_post; a.dgate = dgate;
  a.offset = w_offset; a.eps = eps; a.scale = scale; a.inv_d = 1.f / (float)d;
  a.S = (int)S; a.d = (int)d; a.normalize = normalize != 0;
  return dispatch_bwd<false, true>(a, stream_type, gate_rows, workspace, as_stream(stream));
}

mst_status mst_residual_prenorm_fwd(const void* O, const void* X, int32_t stream_type, int32_t normalize, const void* w_post,
                                    const void* gate, int64_t gate_rows, float scale, const void* w_pre,
                                    float w_offset, float eps, int64_t S, int64_t d, void* Y, void* H,
                                    int8_t* codes_o, uint8_t* exps_o, int8_t* codes_y, uint8_t* exps_y, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  if (!O || !X || !Y || !H) return MST_ERR_NULL_POINTER;
  int64_t gate_groups = 0;
  if ((s = check_gate(gate, gate_rows, scale, S, &gate_groups)) != MST_OK) return s;
  if (!good_type(stream_type) || !good_norm(eps, w_offset) || !both_or_neither(codes_o, exps_o) || !both_or_neither(codes_y, exps_y) ||
      (w_post && !normalize))
    return MST_ERR_BAD_ARGUMENT;
  Operands ops;
  ops.add(O, S * d, 2, false, true);
  ops.add(X, S * d, type_bytes(stream_type), false, true);
  ops.add(w_post, d, 2, false, false);
  ops.add(w_pre, d, 2, false, false);
  ops.add(gate, gate_groups * d, 2, false, false);
  ops.add(Y, S * d, type_bytes(stream_type), true, true);
  ops.add(H, S * d, 2, true, true);
  ops.add(codes_o, S * d, 1, true, true);
  ops.add(exps_o, S * blocks_of_row(d), 1, true, false, 1);
  ops.add(codes_y, S * d, 1, true, true);
  ops.add(exps_y, S * blocks_of_row(d), 1, true, false, 1);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  NormFwd a = {};
  a.X = X; a.O = bf(O); a.w_post = bf(w_post); a.w_pre = bf(w_pre); a.gate = bf(gate);
  a.Y = Y; a.H = static_cast<__bf16*>(H);
  a.codes_o = codes_o; a.exps_o = exps_o; a.codes_y = codes_y; a.exps_y = exps_y;
  a.offset = w_offset; a.eps = eps; a.scale = scale; a.inv_d = 1.f / (float)d;
  a.S = (int)S; a.d = (int)d; a.normalize = normalize != 0;
  a.gate_rows = (int)(gate ? std::min(gate_rows, S) : S);
  a.gates = (int)std::max<int64_t>(gate_groups, 1);
  return stream_type == MST_TYPE_FP32 ? launch_fwd<float, true, true, false>(a, as_stream(stream))
                                      : launch_fwd<__bf16, true, true, false>(a, as_stream(stream));
}

mst_status mst_residual_prenorm_bwd(const void* dH, const void* dres, int32_t stream_type,
                                    const void* Y, const int8_t* codes_y, const uint8_t* exps_y,
                                    const void* O, const int8_t* codes_o, const uint8_t* exps_o,
                                    int32_t normalize, const void* w_post, const void* gate, int64_t gate_rows, float scale,
                                    const void* w_pre, float w_offset, float eps, int64_t S, int64_t d,
                                    void* workspace, size_t workspace_size, void* dY, void* dO,
                                    float* dw_pre, float* dw_post, float* dgate, void* stream) {
  mst_status s = check_shape(S, d);
  if (s != MST_OK) return s;
  int64_t gate_groups = 0;
  if ((s = check_gate(gate, gate_rows, scale, S, &gate_groups)) != MST_OK) return s;
  if (!dH || !dY || !dO || (!Y && !codes_y && !exps_y)) return MST_ERR_NULL_POINTER;
  if (!good_type(stream_type) || !good_norm(eps, w_offset) || !both_or_neither(codes_o, exps_o) || !both_or_neither(codes_y, exps_y) ||
      (O && codes_o) || (Y && codes_y) || (w_post && !normalize) || (dw_post && !w_post) || (dgate && !gate) || (dw_pre && !w_pre))
    return MST_ERR_BAD_ARGUMENT;
  if ((w_pre && !dw_pre) || (w_post && !dw_post) || (gate && !dgate) || ((normalize || gate) && !O && !codes_o)) return MST_ERR_NULL_POINTER;
  const size_t need = workspace_bytes(BwdPlan(S, d, gate_rows, true), d);
  if (!workspace || workspace_size < need) return MST_ERR_WORKSPACE;
  if (!normalize && !gate) O = nullptr, codes_o = nullptr, exps_o = nullptr;
  Operands ops;
  ops.add(dH, S * d, 2, false, true);
  ops.add(dres, S * d, type_bytes(stream_type), false, true);
  ops.add(Y, S * d, type_bytes(stream_type), false, true);
  ops.add(codes_y, S * d, 1, false, true);
  ops.add(exps_y, S * blocks_of_row(d), 1, false, false, 1);
  ops.add(O, S * d, 2, false, true);
  ops.add(codes_o, S * d, 1, false, true);
  ops.add(exps_o, S * blocks_of_row(d), 1, false, false, 1);
  ops.add(w_post, d, 2, false, false);
  ops.add(w_pre, d, 2, false, false);
  ops.add(gate, gate_groups * d, 2, false, false);
  ops.add(workspace, (int64_t)need, 1, true, false, 256);
  ops.add(dY, S * d, type_bytes(stream_type), true, true);
  ops.add(dO, S * d, 2, true, true);
  ops.add(dw_pre, d, 4, true, false);
  ops.add(dw_post, d, 4, true, false);
  ops.add(dgate, gate_groups * d, 4, true, false);
  if ((s = ops.check()) != MST_OK || (s = check_device()) != MST_OK) return s;
  NormBwd a = {};
  a.dH = bf(dH); a.dres = dres; a.X = Y; a.codes_x = codes_y; a.exps_x = exps_y;
  a.O = bf(O); a.codes_o = codes_o; a.exps_o = exps_o;
  a.w_pre = bf(w_pre); a.w_post = bf(w_post); a.gate = bf(gate);
  a.dX = dY; a.dO = static_cast<__bf16*>(dO); a.dw_pre = dw_pre; a.dw_post = dw_post; a.dgate = dgate;
  a.offset = w_offset; a.eps = eps; a.scale = scale; a.inv_d = 1.f / (float)d;
  a.S = (int)S; a.d = (int)d; a.normalize = normalize != 0;
  return dispatch_bwd<true, true>(a, stream_type, gate_rows, workspace, as_stream(stream));
}

}  // extern "C"
