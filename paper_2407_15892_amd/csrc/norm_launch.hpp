// Host side of the launches that the norm library and the MLP library share: how rows are held, the forward kernels, the
// checkpoint's kernels.
#pragma once
#include "../../include/mst_norm.h"
#include "mst_norm_kernels.hpp"

#include <algorithm>
#include <cmath>

namespace mst_norm {

using namespace mst;

// A call whose tensors are more than this reads its inputs past the caches, which cannot hold them beside what else is in there; below
// it a call may find in them what was written just before.  Counted is what it reads and writes, but for the checkpoint that a norm's or a
// residual's forward leaves.  Rows of 4096, bf16, us, through the caches and past them:
//   below   2048 rows: backward of the norm 17.4, 18.4, of the residual 16.1, 17.6, of both 23.6, 24.6; 4096 rows: forward of the norm
//           13.7, 16.7, of the residual 21.2, 23.0, of both 29.8, 32.1; 8192 rows: pack 16.5, 17.7, unpack 15.6, 18.1
//   beyond  12300 rows: backward of the norm 67.0, 63.0, of both 97.4, 90.4; 32768 rows: residual 156.5, 152.1, its backward 124.9, 118.0;
//           131072 rows: pack 269, 252, unpack 258, 250, forward of the norm 437, 433
// Not all of them have their border here: pack gains from 150 MB on (12288 rows 26.4, 25.2), the backward of both norms from 160 (4096 rows
// 40.0, 38.3), unpack from 300 (16400 rows 31.8, 33.3, 24576 rows 49.1, 48.5), and the norm of a checkpoint nowhere (131072 rows 263, 267).
constexpr int64_t kCacheBytes = 192 << 20;

inline mst_status launched() { return hipGetLastError() == hipSuccess ? MST_OK : MST_ERR_LAUNCH; }
inline int64_t blocks_of_row(int64_t d) { return (d + 31) / 32; }
inline bool good_norm(float eps, float offset) { return std::isfinite(eps) && eps >= 0x1p-100f && std::isfinite(offset); }

// How rows are held: chunks of eight columns per lane, and teams of lanes.  A workgroup has as many teams as fit 512 lanes.
struct RowPlan {
  int chunks, teams;
  Team team;
  explicit RowPlan(int64_t d) {
    chunks = d <= 8 * 64 * kNormMaxWaves ? 1 : 2;
    team.lanes = 8;
    while (team.lanes < 64 && team.lanes * 8 < d) team.lanes *= 2;
    team.waves = (int)((d + 8 * 64 * chunks - 1) / (8 * 64 * chunks));
    teams = std::max(1, 512 / (team.lanes * team.waves));
  }
  int threads() const { return team.lanes * team.waves * teams; }
};

// Rows of a team of the forward kernels.  8192 x 4096, us, one and two: rebuilt norm 19.4, 16.7; both norms 59.4, 61.9; of 200 x 4096 4.2, 5.0.
constexpr int fwd_rows(bool res, int chunks) { return chunks == 1 && !res ? 2 : 1; }

template <class T, bool kRes, bool kPre, bool kRebuild, int kPolicy, int kNc>
mst_status launch_fwd_chunks(NormFwd a, const RowPlan& p, hipStream_t st) {
  constexpr int kRb = fwd_rows(kRes, kNc);
  const int64_t kRows = kRb * p.teams;              // of a workgroup
  const int64_t most = (int64_t(1) << 31) / p.threads() * kRows;  // a launch has fewer than 2^32 lanes
  a.team = p.team;
  for (int64_t r = 0; r < a.S; r += most) {
    a.row0 = (int)r;
    hipLaunchKernelGGL((k_norm_fwd<T, kRes, kPre, kRebuild, kPolicy, kNc, kRb>),
                       dim3((unsigned)((std::min(most, a.S - r) + kRows - 1) / kRows)), dim3(p.threads()), 0, st, a);
  }
  return launched();
}
template <class T, bool kRes, bool kPre, bool kRebuild>
mst_status launch_fwd(const NormFwd& a, hipStream_t st) {
  const RowPlan p(a.d);
  const int64_t t = kRebuild ? 1 : sizeof(T), n = (int64_t)a.S * a.d;
  const bool stream = n * (t + (kPre ? 2 : 0) + (kRes ? 2 + t : 0)) > kCacheBytes;
  // Long rows always through the caches.  us, through them and past them, bf16: 2048 x 12288 norm with checkpoint 20.0, 24.8, rebuilt 13.2, 17.8;
  // 8192 x 16384 norm 113.0, 113.4, residual 166, 163, both 254, 252, rebuilt 77, 81; 4096 x 12288 float32, gated: 61.5, 60.4, 98.9, 97.6, both 140, 139.
  if (p.chunks == 2) return launch_fwd_chunks<T, kRes, kPre, kRebuild, 0, 2>(a, p, st);
  return stream ? launch_fwd_chunks<T, kRes, kPre, kRebuild, kNonTemporalAccess, 1>(a, p, st)
                : launch_fwd_chunks<T, kRes, kPre, kRebuild, 0, 1>(a, p, st);
}

// A checkpoint kernel's launches: parts of 16 bytes, fewer than 2^30 of them in one.
template <class T, class Launch> void launch_ckpt(int64_t S, int64_t d, Launch launch) {
  constexpr uint32_t kPer = kCkptThreads * kCkptParts;                // of a workgroup
  const FastDiv per_row((uint32_t)(32 / kCkptPart<T> * blocks_of_row(d)));
  const int64_t most = (int64_t(1) << 30) / per_row.d;
  for (int64_t r = 0, n; r < S; r += n) {
    n = std::min(S - r, most);
    const uint32_t parts = (uint32_t)n * per_row.d;
    launch(r, dim3((parts + kPer - 1) / kPer), per_row, parts);
  }
}
template <class T> void launch_pack(const T* X, int64_t S, int64_t d, int8_t* codes, uint8_t* exps, hipStream_t st) {
  const auto kernel = S * d * (int64_t)(sizeof(T) + 1) > kCacheBytes ? k_ckpt_pack<T, true> : k_ckpt_pack<T, false>;
  launch_ckpt<T>(S, d, [&](int64_t r, dim3 grid, FastDiv per_row, uint32_t parts) {
    hipLaunchKernelGGL(kernel, grid, dim3(kCkptThreads), 0, st, X + r * d, per_row, parts, (int)d, codes + r * d, exps + r * blocks_of_row(d));
  });
}
template <class T> void launch_unpack(const int8_t* codes, const uint8_t* exps, int64_t S, int64_t d, T* X, hipStream_t st) {
  const auto kernel = S * d * (int64_t)(sizeof(T) + 1) > kCacheBytes ? k_ckpt_unpack<T, true> : k_ckpt_unpack<T, false>;
  launch_ckpt<T>(S, d, [&](int64_t r, dim3 grid, FastDiv per_row, uint32_t parts) {
    hipLaunchKernelGGL(kernel, grid, dim3(kCkptThreads), 0, st, codes + r * d, exps + r * blocks_of_row(d), per_row, parts, (int)d, X + r * d);
  });
}

}  // namespace mst_norm
