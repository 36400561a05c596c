// Device kernels between the mini-sequence blocks (gfx950): norms, the gated residual, their gradients, and 8-bit
// checkpoints.  The formulas are in include/mst_norm.h.
//
//   k_ckpt_pack, k_ckpt_unpack   the checkpoint alone
//   k_norm_fwd                   norm before a block, residual after it, or both
//   k_norm_bwd                   their gradients; per workgroup sums over its rows for those of weights and gates
//   k_norm_reduce                these sums over the workgroups, in fixed order
//
// All of them move data and compute little, so a row is read once: a workgroup holds its columns in registers (8 adjacent ones
// per lane and chunk of 8 * threads: 16 bytes of bf16), sums over the row go through DPP and LDS, and what is needed
// of the row is written from the registers.  Four adjacent lanes hold the 32 columns of a checkpoint's block, whose largest
// magnitude two quad permutations find.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace mst {

typedef float norm_f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned norm_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned norm_u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 norm_bf16x2 __attribute__((ext_vector_type(2)));
typedef float norm_f32x2 __attribute__((ext_vector_type(2)));

// Eight adjacent entries of a row as they are in memory.
template <class T> struct Eight;
template <> struct Eight<__bf16> {
  norm_u32x4 u = {0, 0, 0, 0};
  __device__ void load(const __bf16* p) { u = *reinterpret_cast<const norm_u32x4*>(p); }
  __device__ void store(__bf16* p) const { *reinterpret_cast<norm_u32x4*>(p) = u; }
  __device__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  __device__ void set(const float (&v)[8]) {      // to nearest, ties to even
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const norm_f32x2 pair = {v[2 * i], v[2 * i + 1]};
      u[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(pair, norm_bf16x2));
    }
  }
};
template <> struct Eight<float> {
  norm_f32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
  __device__ void load(const float* p) {
    a = *reinterpret_cast<const norm_f32x4*>(p);
    b = *reinterpret_cast<const norm_f32x4*>(p + 4);
  }
  __device__ void store(float* p) const {
    *reinterpret_cast<norm_f32x4*>(p) = a;
    *reinterpret_cast<norm_f32x4*>(p + 4) = b;
  }
  __device__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  }
  __device__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = v[i]; b[i] = v[4 + i]; }
  }
};

// A signed byte of a word as a float, in one instruction (which the compiler does not find).
template <int kByte> __device__ __forceinline__ float signed_byte(unsigned u) {
  float f;
  if (kByte == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(u));
  if (kByte == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(u));
  if (kByte == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(u));
  if (kByte == 3) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(u));
  return f;
}

// Eight entries of a checkpoint.
struct EightCodes {
  norm_u32x2 c = {0, 0};
  unsigned e = 0;
  __device__ void load(const int8_t* codes, const uint8_t* exp) {
    c = *reinterpret_cast<const norm_u32x2*>(codes);
    e = *exp;
  }
  __device__ void get(float (&v)[8]) const {
    // 2^(e - 127): of 0 a subnormal, of 255 NaN
    const float scale = __uint_as_float(max(e << 23 | ((e + 1) >> 8) << 22, 0x00400000u));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[4 * i] = signed_byte<0>(c[i]) * scale;
      v[4 * i + 1] = signed_byte<1>(c[i]) * scale;
      v[4 * i + 2] = signed_byte<2>(c[i]) * scale;
      v[4 * i + 3] = signed_byte<3>(c[i]) * scale;
    }
  }
};

template <int kCtrl> __device__ __forceinline__ unsigned dpp_u32(unsigned x) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, true);
}
template <int kCtrl> __device__ __forceinline__ float dpp_f32(float x) { return __uint_as_float(dpp_u32<kCtrl>(__float_as_uint(x))); }
constexpr int kQuadSwap1 = 0xB1, kQuadSwap2 = 0x4E;                 // quad_perm [1 0 3 2], [2 3 0 1]
constexpr int kHalfMirror = 0x141, kMirror = 0x140;                 // within 8 and 16 lanes

// Codes of eight entries and the exponent byte of their block of 32, whose other entries are in the other lanes of the quad
// (all four lanes call this; lanes behind the row's end hold zeros).  The least scale whose product with 127.5 is more than
// the largest magnitude m * 2^e: 2^(e - 6), or 2^(e - 5) from m = 127.5 / 64 = 1 + 127 / 128 on, where adding the last bit of
// that mantissa carries into the exponent.  x / scale + 1.5 * 2^23 rounds to the nearest integer, ties to even, and has its
// two's complement in the low byte.  Measured as integers magnitudes order NaN above infinity above all else.
struct Packed { norm_u32x2 codes; unsigned exp; };
__device__ __forceinline__ Packed pack_eight(const float (&v)[8]) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned m = __float_as_uint(v[i]) & 0x7fffffffu;
    top = top > m ? top : m;
  }
  unsigned o = dpp_u32<kQuadSwap1>(top);
  top = top > o ? top : o;
  o = dpp_u32<kQuadSwap2>(top);
  top = top > o ? top : o;
  const unsigned E = (top + 0x10000u) >> 23;
  Packed p;
  p.exp = E >= 255 ? 255 : max(E, 6u) - 6;
  const float inverse = __uint_as_float((254u - p.exp) << 23);
  unsigned b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(v[i], inverse, 12582912.f));
#pragma unroll
  for (int i = 0; i < 2; ++i)      // the low bytes of four words
    p.codes[i] = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u) | __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000c0cu);
  return p;
}

// ---- the checkpoint alone ------------------------------------------------------------------------------------------------

// n / d for 0 <= n < 2^31 by a multiplication (m = floor(2^(31 + l) / d) + 1, 2^l >= d).
struct FastDiv {
  uint32_t m, shift, d;
  FastDiv() = default;
  explicit FastDiv(uint32_t by) : d(by) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < by) ++l;
    shift = 31 + l;
    m = (uint32_t)((uint64_t(1) << shift) / by + 1);
  }
  __host__ __device__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> shift); }
};

constexpr int kCkptThreads = 256;

// One lane per eight entries; a row takes a whole number of quads, so that a quad is a block.
template <class T>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_pack(const T* X, FastDiv per_row, uint32_t slots, int d, int8_t* codes, uint8_t* exps) {
  const uint32_t n = blockIdx.x * kCkptThreads + threadIdx.x;
  const uint32_t row = per_row(n < slots ? n : 0), in_row = n - row * per_row.d;
  const bool on = n < slots && (int)in_row * 8 < d;
  Eight<T> x;
  if (on) x.load(X + (size_t)row * d + in_row * 8);
  float v[8];
  x.get(v);
  const Packed p = pack_eight(v);
  if (!on) return;
  *reinterpret_cast<norm_u32x2*>(codes + (size_t)row * d + in_row * 8) = p.codes;
  if (threadIdx.x % 4 == 0) exps[(n >> 2)] = (uint8_t)p.exp;
}

template <class T>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_unpack(const int8_t* codes, const uint8_t* exps, FastDiv per_row, uint32_t slots, int d, T* X) {
  const uint32_t n = blockIdx.x * kCkptThreads + threadIdx.x;
  if (n >= slots) return;
  const uint32_t row = per_row(n), in_row = n - row * per_row.d;
  if ((int)in_row * 8 >= d) return;
  const size_t at = (size_t)row * d + in_row * 8;
  EightCodes c;
  c.load(codes + at, exps + (n >> 2));
  float v[8];
  c.get(v);
  Eight<T> x;
  x.set(v);
  x.store(X + at);
}

// ---- sums over a row -----------------------------------------------------------------------------------------------------

// Lanes that hold a row together (a team): 8, 16 or 32 of a wave for short rows, else `waves` whole waves.
struct Team {
  int lanes, waves;        // lanes: of one wave
  __device__ int threads() const { return lanes * waves; }
};

template <int kN> __device__ __forceinline__ void add_all(float (&v)[kN], const float (&o)[kN]) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] += o[i];
}
template <int kCtrl, int kN> __device__ __forceinline__ void add_dpp(float (&v)[kN]) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] += dpp_f32<kCtrl>(v[i]);
}
__device__ __forceinline__ float lane_of(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }

constexpr int kNormMaxWaves = 16;

// A barrier that waits for this wave's LDS accesses, but not for global loads that are on their way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Sums of kN values over a team, in every one of its lanes, always in the same order.  All of the workgroup calls it.  Two
// buffers in turn: one barrier a sum, none where a team is within a wave.
template <int kN> struct RowSums {
  float (*lds)[kNormMaxWaves][kN];       // [2]
  const Team team;
  int turn = 0;
  __device__ RowSums(float (*buffers)[kNormMaxWaves][kN], Team t) : lds(buffers), team(t) {}
  __device__ __forceinline__ void operator()(float (&v)[kN]) {
    add_dpp<kQuadSwap1>(v);
    add_dpp<kQuadSwap2>(v);
    add_dpp<kHalfMirror>(v);
    if (team.lanes == 8) return;
    add_dpp<kMirror>(v);
    if (team.lanes == 16) return;
    if (team.lanes == 32) {
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v[i]), 0x401f));   // lane ^ 16
      return;
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = (lane_of(v[i], 0) + lane_of(v[i], 16)) + (lane_of(v[i], 32) + lane_of(v[i], 48));
    if (team.waves == 1) return;
    const int wave = threadIdx.x / 64, first = wave / team.waves * team.waves;
    float (*const at)[kN] = lds[turn];
    turn ^= 1;
    if (threadIdx.x % 64 == 0) {
#pragma unroll
      for (int i = 0; i < kN; ++i) at[wave][i] = v[i];
    }
    lds_barrier();
    const int from = threadIdx.x % (team.waves > 8 ? 16 : 8);      // each 8 or 16 lanes read the waves' sums and add them up
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float x = at[(first + from) % kNormMaxWaves][i];
      v[i] = from < team.waves ? x : 0.f;
    }
    add_dpp<kQuadSwap1>(v);
    add_dpp<kQuadSwap2>(v);
    add_dpp<kHalfMirror>(v);
    if (team.waves > 8) add_dpp<kMirror>(v);
  }
};

// ---- forward -------------------------------------------------------------------------------------------------------------

struct NormFwd {
  const void* X;                   // stream type; without kRes NULL where codes_x stand for it
  const __bf16* O;
  const __bf16 *w_pre, *w_post;    // NULL: ones
  const __bf16* gate;              // NULL: ones
  void* Y;
  __bf16* H;
  const int8_t* codes_x; const uint8_t* exps_x;
  int8_t* codes_o; uint8_t* exps_o;
  int8_t* codes_y; uint8_t* exps_y;      // of Y, or without kRes of X
  float offset, eps, scale, inv_d;
  int S, d, normalize, gate_rows;
  int row0;                        // first row of the launch
  Team team;
};

// The weights of eight columns.
__device__ __forceinline__ void weights(const __bf16* w, float offset, int col, bool on, float (&v)[8]) {
  Eight<__bf16> e;
  if (w) {
    if (on) e.load(w + col);
    e.get(v);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = offset + (w ? v[i] : 1.f);
}

__device__ __forceinline__ void store_packed(const Packed& p, int8_t* codes, uint8_t* exps, size_t row, int d, int col) {
  *reinterpret_cast<norm_u32x2*>(codes + row * d + col) = p.codes;
  if (threadIdx.x % 4 == 0) exps[row * ((d + 31) / 32) + col / 32] = (uint8_t)p.exp;
}

// kRb rows per team, kNc chunks of 8 columns per lane.
template <class T, bool kRes, bool kPre, bool kRebuild, int kNc, int kRb>
__global__ __launch_bounds__(1024) void k_norm_fwd(const NormFwd a) {
  __shared__ float lds[2][kNormMaxWaves][kRb];
  RowSums<kRb> row_sums(lds, a.team);
  const int threads = a.team.threads(), lane = threadIdx.x % threads, d = a.d;
  const int r0 = a.row0 + (blockIdx.x * (blockDim.x / threads) + threadIdx.x / threads) * kRb;
  const T* const X = static_cast<const T*>(a.X);
  float x[kRb][kNc][8];
  Eight<T> raw[kRb][kNc];
  Eight<__bf16> o[kRb][kNc];
  EightCodes c[kRb][kNc];
#pragma unroll
  for (int r = 0; r < kRb; ++r)
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      const int col = (k * threads + lane) * 8;
      const size_t at = (size_t)(r0 + r) * d + col;
      if (r0 + r < a.S && col < d) {
        if (kRebuild) c[r][k].load(a.codes_x + at, a.exps_x + (size_t)(r0 + r) * ((d + 31) / 32) + col / 32);
        else raw[r][k].load(X + at);
        if (kRes) o[r][k].load(a.O + at);
      }
    }
  if (kRes) {
    float rstd[kRb];
    if (a.normalize) {
#pragma unroll
      for (int r = 0; r < kRb; ++r) {
        rstd[r] = 0.f;
#pragma unroll
        for (int k = 0; k < kNc; ++k) {
          float v[8];
          o[r][k].get(v);
#pragma unroll
          for (int i = 0; i < 8; ++i) rstd[r] = fmaf(v[i], v[i], rstd[r]);
        }
      }
      row_sums(rstd);
#pragma unroll
      for (int r = 0; r < kRb; ++r) rstd[r] = rsqrtf(fmaf(rstd[r], a.inv_d, a.eps));
    }
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      const int col = (k * threads + lane) * 8;
      const bool on = col < d;
      float w[8];
      if (a.normalize) weights(a.w_post, a.offset, col, on, w);
#pragma unroll
      for (int r = 0; r < kRb; ++r) {
        const size_t row = r0 + r;
        const bool here = on && r0 + r < a.S;
        float v[8], base[8];
        o[r][k].get(v);
        if (a.codes_o) {
          const Packed p = pack_eight(v);
          if (here) store_packed(p, a.codes_o, a.exps_o, row, d, col);
        }
        raw[r][k].get(base);
        float g[8];
        weights(a.gate ? a.gate + (size_t)((unsigned)(r0 + r) / (unsigned)a.gate_rows) * d : nullptr, 0.f, col, here, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float n = a.normalize ? v[i] * rstd[r] * w[i] : v[i];
          x[r][k][i] = fmaf(a.scale * g[i], n, base[i]);
        }
        raw[r][k].set(x[r][k]);
        if (here) raw[r][k].store(static_cast<T*>(a.Y) + row * d + col);
        if (kPre && a.codes_y) {
          raw[r][k].get(base);
          const Packed p = pack_eight(base);
          if (here) store_packed(p, a.codes_y, a.exps_y, row, d, col);
        }
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < kRb; ++r)
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        if (kRebuild) c[r][k].get(x[r][k]);
        else raw[r][k].get(x[r][k]);
        if (!kRebuild && a.codes_y) {
          const int col = (k * threads + lane) * 8;
          const Packed p = pack_eight(x[r][k]);
          if (r0 + r < a.S && col < d) store_packed(p, a.codes_y, a.exps_y, r0 + r, d, col);
        }
      }
  }
  if (!kPre) return;
  float rstd[kRb];
#pragma unroll
  for (int r = 0; r < kRb; ++r) {
    rstd[r] = 0.f;
#pragma unroll
    for (int k = 0; k < kNc; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) rstd[r] = fmaf(x[r][k][i], x[r][k][i], rstd[r]);
  }
  row_sums(rstd);
#pragma unroll
  for (int r = 0; r < kRb; ++r) rstd[r] = rsqrtf(fmaf(rstd[r], a.inv_d, a.eps));
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    const int col = (k * threads + lane) * 8;
    float w[8];
    weights(a.w_pre, a.offset, col, col < d, w);
#pragma unroll
    for (int r = 0; r < kRb; ++r) {
      if (r0 + r >= a.S || col >= d) continue;
      float h[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = x[r][k][i] * rstd[r] * w[i];
      Eight<__bf16> e;
      e.set(h);
      e.store(a.H + (size_t)(r0 + r) * d + col);
    }
  }
}

// ---- backward ------------------------------------------------------------------------------------------------------------

struct NormBwd {
  const __bf16* dH;
  const void *dres, *dY;           // stream type; dres may be NULL, dY is read without kPre
  const void* X; const int8_t* codes_x; const uint8_t* exps_x;      // X (between blocks: Y), or its checkpoint
  const __bf16* O; const int8_t* codes_o; const uint8_t* exps_o;    // O or its checkpoint, or neither
  const __bf16 *w_pre, *w_post, *gate;
  void* dX;                        // with kPre
  __bf16* dO;
  float *dw_pre, *dw_post, *dgate; // NULL: not wanted
  float *part_pre, *part_post;     // [workgroups][d] each
  float offset, eps, scale, inv_d;
  int S, d, normalize;
  int gate_rows;                   // without a gate S
  int share;                       // workgroups that share a row of the gate (not kWhole)
  int rows;                        // that a team takes in turn
  Team team;
};

// Some rows of a tensor as a buffer: what lies behind them, and a tensor that is not there, reads as zeros and takes no
// stores.  Without branches around loads and stores the compiler knows how many are under way, and waits for the ones it needs.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const void* p, int64_t from, int rows, int row_bytes) {
  const char* const at = static_cast<const char*>(p) + from * row_bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, p ? rows * row_bytes : 0, 0x00020000);
}
// Offset in entries of a lane that has no columns: behind those rows (less than 2^29 entries) in bytes of 1, 2 or 4.
constexpr uint32_t kNoColumn = 1u << 29;
// Rows whose loads are under way while one is summed up.
template <class T> constexpr int rows_ahead(bool pre, bool res, int chunks) { return pre && !res && chunks == 1 && sizeof(T) == 2 ? 2 : 1; }

constexpr int kNonTemporalAccess = 2;         // cache policy of buffer loads and stores

template <int kPolicy, class T> __device__ __forceinline__ void load_eight(Eight<T>& e, __amdgpu_buffer_rsrc_t rows, uint32_t at) {
  const uint32_t byte = at * (uint32_t)sizeof(T);
  if constexpr (sizeof(T) == 2) {
    e.u = __builtin_bit_cast(norm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, byte, 0, kPolicy));
  } else {
    e.a = __builtin_bit_cast(norm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, byte, 0, kPolicy));
    e.b = __builtin_bit_cast(norm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, byte + 16, 0, kPolicy));
  }
}
template <class T> __device__ __forceinline__ void store_eight(const Eight<T>& e, __amdgpu_buffer_rsrc_t rows, uint32_t at) {
  const uint32_t byte = at * (uint32_t)sizeof(T);
  if constexpr (sizeof(T) == 2) {
    __builtin_amdgcn_raw_buffer_store_b128(e.u, rows, byte, 0, kNonTemporalAccess);
  } else {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(norm_u32x4, e.a), rows, byte, 0, kNonTemporalAccess);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(norm_u32x4, e.b), rows, byte + 16, 0, kNonTemporalAccess);
  }
}

// A row's eight entries: the tensor's, or those of its checkpoint.
template <class T, bool kCheckpoint, int kPolicy> struct Source {
  Eight<T> e;
  __device__ void load(__amdgpu_buffer_rsrc_t rows, __amdgpu_buffer_rsrc_t, uint32_t at, uint32_t) { load_eight<kPolicy>(e, rows, at); }
  __device__ void get(float (&v)[8]) const { e.get(v); }
};
template <class T, int kPolicy> struct Source<T, true, kPolicy> {
  EightCodes e;
  __device__ void load(__amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t exps, uint32_t at, uint32_t block) {
    e.c = __builtin_bit_cast(norm_u32x2, __builtin_amdgcn_raw_buffer_load_b64(codes, at, 0, kPolicy));
    e.e = __builtin_amdgcn_raw_buffer_load_b8(exps, block, 0, kPolicy);
  }
  __device__ void get(float (&v)[8]) const { e.get(v); }
};

// dw_post and dgate of kN columns from t = sum of dY * N / w_post over the rows of a row of the gate (dw_post: if it is the
// only one, or there is no gate).
__device__ __forceinline__ float post_weight(const NormBwd& a, int col) {
  return a.scale * (a.normalize ? a.offset + (a.w_post ? (float)a.w_post[col] : 1.f) : 1.f);
}
__device__ __forceinline__ float gate_factor(const NormBwd& a, int group, int col) {
  return a.scale * (a.gate ? (float)a.gate[(size_t)group * a.d + col] : 1.f);
}
template <int kN> __device__ __forceinline__ void finish_post(const NormBwd& a, int col, const float* t) {
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    if (a.dw_post) a.dw_post[col + i] = gate_factor(a, 0, col + i) * t[i];
    if (a.dgate) a.dgate[col + i] = post_weight(a, col + i) * t[i];
  }
}

// A team takes `rows` rows in turn, the next one's loads on their way while it computes; its lanes keep the sums over them
// for their columns.
//   kWhole = false  `share` workgroups have the rows of one row of the gate (all rows without a gate), adjacent rows in
//                   adjacent teams: memory is passed through in a few streams.  Sums of dY * N, without the gate, to the workspace.
//   kWhole = true   for many short rows of gates: a team has all rows of one, then those of another; it writes their gradient
//                   and sums up dw_post.
// With x the row of X, q its rstd, a = dH * ~w: the gradient is dres + q a - x q^3 sum(a x) / d; likewise for O with
// b = dY * f, f = scale * gate * ~w_post.  One sum over the row waits for another where both norms are there.
template <class T, bool kPre, bool kRes, bool kWhole, bool kCkptX, bool kCkptO, int kPolicy, int kNc>
__global__ __launch_bounds__(1024) void k_norm_bwd(const NormBwd a) {
  constexpr int kFirst = (kPre ? 2 : 0) + (kRes ? kPre ? 1 : 2 : 0);   // sums over a row that wait for nothing
  __shared__ float lds1[2][kNormMaxWaves][kFirst], lds2[2][kNormMaxWaves][1];
  extern __shared__ float lds_columns[];
  RowSums<kFirst> first_sums(lds1, a.team);
  RowSums<1> second_sum(lds2, a.team);
  const int d = a.d, blocks = (d + 31) / 32, threads = a.team.threads(), lane = threadIdx.x % threads;
  const int teams = blockDim.x / threads, in_block = threadIdx.x / threads;
  // The workgroup's rows at a time: those of its teams, `apart` rows from each other, the first at `row`.
  const int apart = kWhole ? a.gate_rows : 1;
  int group = kWhole ? (int)blockIdx.x * teams : (int)blockIdx.x / a.share;      // the gate's row (of the first team)
  const int end = kWhole ? a.S : (int)min((int64_t)(group + 1) * a.gate_rows, (int64_t)a.S);
  int64_t row = (int64_t)group * a.gate_rows + (kWhole ? 0 : (int64_t)(blockIdx.x % a.share) * teams), next = row;
  int in_group = 0, next_in_group = 0;             // kWhole: rows of the gate's row that are done
  auto advance = [&](int64_t& r, int& done) {
    if (kWhole) {
      ++r;
      if (++done == a.gate_rows) {
        done = 0;
        r += ((int64_t)gridDim.x * teams - 1) * a.gate_rows;
      }
    } else {
      r += (int64_t)a.share * teams;
    }
  };
  float acc_pre[kNc][8] = {}, acc_group[kNc][8] = {}, acc_post[kNc][8] = {};
  float w[kNc][8], f[kNc][8];
  auto column = [&](int k) { return (k * threads + lane) * 8; };
  auto load_f = [&](int k, int g, bool on) {
    const int col = column(k);
    weights(a.gate ? a.gate + (size_t)g * d : nullptr, 0.f, col, on && col < d, f[k]);
    float wo[8];
    weights(a.normalize ? a.w_post : nullptr, a.normalize ? a.offset : 0.f, col, col < d, wo);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[k][i] *= a.scale * wo[i];
  };
  uint32_t at[kNc], block[kNc];
  constexpr int kAhead = rows_ahead<T>(kPre, kRes, kNc);
  Eight<__bf16> dh_next[kAhead][kNc];
  Source<T, kCkptX, kPolicy> x_next[kAhead][kNc];
  Eight<T> dy_next[kAhead][kNc];
  Source<__bf16, kCkptO, kPolicy> o_next[kAhead][kNc];
  auto rows_at = [&](int64_t r) { return (int)max((int64_t)0, min((int64_t)(teams - 1) * apart + 1, end - r)); };
  auto load = [&](int slot) {
    const int rows = rows_at(next);
    const __amdgpu_buffer_rsrc_t dy_rows = rows_of(kPre ? a.dres : a.dY, next, rows, (int)sizeof(T) * d);
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      if (kPre) {
        load_eight<kPolicy>(dh_next[slot][k], rows_of(a.dH, next, rows, 2 * d), at[k]);
        x_next[slot][k].load(kCkptX ? rows_of(a.codes_x, next, rows, d) : rows_of(a.X, next, rows, (int)sizeof(T) * d),
                       rows_of(a.exps_x, next, rows, blocks), at[k], block[k]);
      }
      load_eight<kPolicy>(dy_next[slot][k], dy_rows, at[k]);
      if (kRes)
        o_next[slot][k].load(kCkptO ? rows_of(a.codes_o, next, rows, d) : rows_of(a.O, next, rows, 2 * d), rows_of(a.exps_o, next, rows, blocks),
                       at[k], block[k]);
    }
    advance(next, next_in_group);
  };
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    const bool on = column(k) < d;
    at[k] = on ? in_block * apart * d + column(k) : kNoColumn;
    block[k] = on ? in_block * apart * blocks + column(k) / 32 : kNoColumn;
    if (kPre) weights(a.w_pre, a.offset, column(k), on, w[k]);
    if (kRes && !kWhole) load_f(k, group, true);
  }
#pragma unroll
  for (int slot = 0; slot < kAhead; ++slot) load(slot);
  auto one_row = [&](int slot) {
    float dh[kNc][8], x[kNc][8], dy[kNc][8], o[kNc][8];
    float sums[kFirst];
#pragma unroll
    for (int i = 0; i < kFirst; ++i) sums[i] = 0.f;
    if (kWhole && in_group == 0) {
#pragma unroll
      for (int k = 0; k < kNc; ++k) load_f(k, group + in_block, row + (int64_t)in_block * apart < end);
    }
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      dy_next[slot][k].get(dy[k]);
      if (kPre) {
        x_next[slot][k].get(x[k]);
        dh_next[slot][k].get(dh[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sums[0] = fmaf(x[k][i], x[k][i], sums[0]);
          sums[1] = fmaf(dh[k][i] * w[k][i], x[k][i], sums[1]);
        }
      }
      if (kRes) {
        o_next[slot][k].get(o[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sums[kPre ? 2 : 0] = fmaf(o[k][i], o[k][i], sums[kPre ? 2 : 0]);
          if (!kPre) sums[1] = fmaf(dy[k][i] * f[k][i], o[k][i], sums[1]);
        }
      }
    }
    load(slot);
    const int rows = rows_at(row);
    if (kPre || a.normalize) first_sums(sums);
    float post[1] = {kPre ? 0.f : sums[1]};      // sum of b * O
    if (kPre) {
      const float q = rsqrtf(fmaf(sums[0], a.inv_d, a.eps)), c = -q * q * q * sums[1] * a.inv_d;
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = dh[k][i] * q;
          acc_pre[k][i] = fmaf(u, x[k][i], acc_pre[k][i]);
          dy[k][i] = fmaf(u, w[k][i], dy[k][i]);
          dy[k][i] = fmaf(x[k][i], c, dy[k][i]);
          if (kRes) post[0] = fmaf(dy[k][i] * f[k][i], o[k][i], post[0]);
        }
        Eight<T> e;
        e.set(dy[k]);
        store_eight(e, rows_of(a.dX, row, rows, (int)sizeof(T) * d), at[k]);
      }
    }
    if (kRes) {
      if (kPre && a.normalize) second_sum(post);
      const float q = a.normalize ? rsqrtf(fmaf(sums[kPre ? 2 : 0], a.inv_d, a.eps)) : 1.f;
      const float c = a.normalize ? -q * q * q * post[0] * a.inv_d : 0.f;
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        float out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = dy[k][i] * q;
          out[i] = fmaf(o[k][i], c, u * f[k][i]);
          acc_group[k][i] = fmaf(u, o[k][i], acc_group[k][i]);
        }
        Eight<__bf16> e;
        e.set(out);
        store_eight(e, rows_of(a.dO, row, rows, 2 * d), at[k]);
      }
      const int64_t mine = row + (int64_t)in_block * apart;
      if (kWhole && (in_group == a.gate_rows - 1 || mine == end - 1) && mine < end) {      // the last row of its row of the gate
#pragma unroll
        for (int k = 0; k < kNc; ++k) {
          const int col = column(k);
          if (col >= d) continue;
          Eight<float> e;
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            acc_post[k][i] = fmaf(gate_factor(a, group + in_block, col + i), acc_group[k][i], acc_post[k][i]);
            v[i] = post_weight(a, col + i) * acc_group[k][i];
            acc_group[k][i] = 0.f;
          }
          e.set(v);
          e.store(a.dgate + (size_t)(group + in_block) * d + col);
        }
      }
    }
    advance(row, in_group);
    if (kWhole && in_group == 0) group += gridDim.x * teams;
  };
  for (int i_row = 0; i_row < a.rows; i_row += kAhead) {         // as often in every team, for the barriers; zeros behind the last row
#pragma unroll
    for (int slot = 0; slot < kAhead; ++slot) one_row(slot);
  }
  // the teams' sums, then to the workspace, or where they belong if this is the only workgroup
  auto add_teams = [&](const float (&acc)[kNc][8], auto put) {
    if (teams == 1) {
#pragma unroll
      for (int k = 0; k < kNc; ++k)
        if (column(k) < d) put(column(k), acc[k], std::integral_constant<int, 8>());
      return;
    }
    __syncthreads();
    if (column(0) < d) {
#pragma unroll
      for (int i = 0; i < 8; ++i) lds_columns[in_block * d + column(0) + i] = acc[0][i];
    }
    __syncthreads();
    for (int col = threadIdx.x; col < d; col += blockDim.x) {
      float sum[1] = {0.f};
      for (int t = 0; t < teams; ++t) sum[0] += lds_columns[t * d + col];
      put(col, sum, std::integral_constant<int, 1>());
    }
  };
  auto store = [&](float* to) {
    return [=](int col, const float* v, auto n) {
#pragma unroll
      for (int i = 0; i < decltype(n)::value; ++i) to[col + i] = v[i];
    };
  };
  const bool alone = gridDim.x == 1;
  if (kPre && a.dw_pre) add_teams(acc_pre, store(alone ? a.dw_pre : a.part_pre + (size_t)blockIdx.x * d));
  if (kRes && kWhole && a.dw_post) add_teams(acc_post, store(alone ? a.dw_post : a.part_post + (size_t)blockIdx.x * d));
  if (kRes && !kWhole && (a.dw_post || a.dgate)) {
    if (alone) add_teams(acc_group, [&](int col, const float* v, auto n) { finish_post<decltype(n)::value>(a, col, v); });
    else add_teams(acc_group, store(a.part_post + (size_t)blockIdx.x * d));
  }
}

// Sums of the workgroups' sums (n of them): blockIdx.y = 0 dw_pre; 1 dw_post, each times its row of the gate if the
// workgroups have not done that (and the gradient of a single row of gates); from 2 on the gradients of several rows of gates, `share` sums
// each.  A workgroup takes 32 columns (a cache line of each sum): 8 lanes of four, and 128 groups of 8 lanes; of these `slices`
// (a power of two) share out the sums of a result, and are added up in one order.
constexpr int kReduceThreads = 1024, kReduceCols = 32, kReduceSlices = kReduceThreads / 8;
__global__ __launch_bounds__(kReduceThreads) void k_norm_reduce(const NormBwd a, int n, int whole, int gate_slices) {
  __shared__ norm_f32x4 lds[kReduceSlices / 8][8];
  const int lane = threadIdx.x % 8, slice = threadIdx.x / 8, d = a.d;
  const int col = blockIdx.x * kReduceCols + lane * 4;
  const int gates = a.dgate && !whole ? n / a.share : 0;
  const bool one_gate = gates == 1;
  int slices = kReduceSlices, first = 0, count = n, group = 0;
  const float* part = blockIdx.y == 0 ? a.part_pre : a.part_post;
  if (blockIdx.y == 0 ? !a.dw_pre : blockIdx.y == 1 && !a.dw_post && !one_gate) return;
  if (blockIdx.y >= 2) {
    slices = gate_slices;
    group = (blockIdx.y - 2) * (kReduceSlices / slices) + slice / slices;
    first = group * a.share;
    count = group < gates ? a.share : 0;
  }
  const bool weighted = blockIdx.y == 1 && gates > 1;
  norm_f32x4 sum = {0, 0, 0, 0};
  if (col < d) {
#pragma unroll 4
    for (int p = slice % slices; p < count; p += slices) {
      norm_f32x4 v = *reinterpret_cast<const norm_f32x4*>(part + (size_t)(first + p) * d + col);
      if (weighted) {
        for (int i = 0; i < 4; ++i) v[i] *= gate_factor(a, p / a.share, col + i);
      }
      sum += v;
    }
  }
#pragma unroll
  for (int x = 8; x < 64; x *= 2) {            // the eight slices of a wave
    if (x >= slices * 8) break;
    norm_f32x4 o;
    for (int i = 0; i < 4; ++i) o[i] = __shfl_xor(sum[i], x);
    sum += o;
  }
  if (slices > 8) {
    if (slice % 8 == 0) lds[slice / 8][lane] = sum;
    __syncthreads();
    if (slice % slices == 0) {
      for (int s = 1; s < slices / 8; ++s) sum += lds[slice / 8 + s][lane];
    }
  }
  if (slice % slices || col >= d || count == 0) return;
  float t[4];
  for (int i = 0; i < 4; ++i) t[i] = sum[i];
  if (blockIdx.y == 1 && !whole && !weighted) {
    finish_post<4>(a, col, t);
    return;
  }
  float* const to = blockIdx.y == 0 ? a.dw_pre : blockIdx.y == 1 ? a.dw_post : a.dgate + (size_t)group * d;
  for (int i = 0; i < 4; ++i) to[col + i] = blockIdx.y < 2 ? t[i] : post_weight(a, col + i) * t[i];
}

}  // namespace mst
