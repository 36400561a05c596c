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

__device__ __forceinline__ float wave_sum(float x) {      // of all 64 lanes, in all of them, in one order
  x += dpp_f32<kQuadSwap1>(x);
  x += dpp_f32<kQuadSwap2>(x);
  x += dpp_f32<kHalfMirror>(x);
  x += dpp_f32<kMirror>(x);
  const int b = __float_as_int(x);
  return (__int_as_float(__builtin_amdgcn_readlane(b, 0)) + __int_as_float(__builtin_amdgcn_readlane(b, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(b, 32)) + __int_as_float(__builtin_amdgcn_readlane(b, 48)));
}

constexpr int kNormMaxWaves = 16;

// Sums of kN values over the workgroup, in every lane.  Two buffers in turn: one barrier a sum.
template <int kN> struct RowSums {
  float (*lds)[kNormMaxWaves][kN];       // [2]
  int turn = 0;
  __device__ explicit RowSums(float (*buffers)[kNormMaxWaves][kN]) : lds(buffers) {}
  __device__ __forceinline__ void operator()(float (&v)[kN]) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = wave_sum(v[i]);
    const int waves = blockDim.x / 64;
    if (waves == 1) return;
    float (*const at)[kN] = lds[turn];
    turn ^= 1;
    if (threadIdx.x % 64 == 0) {
#pragma unroll
      for (int i = 0; i < kN; ++i) at[threadIdx.x / 64][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = 0.f;
    for (int w = 0; w < waves; ++w) {
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += at[w][i];
    }
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

// kRb rows per workgroup, kNc chunks of 8 columns per lane.
template <class T, bool kRes, bool kPre, bool kRebuild, int kNc, int kRb>
__global__ __launch_bounds__(1024) void k_norm_fwd(const NormFwd a) {
  __shared__ float lds[2][kNormMaxWaves][kRb];
  RowSums<kRb> row_sums(lds);
  const int r0 = a.row0 + blockIdx.x * kRb, d = a.d;
  const T* const X = static_cast<const T*>(a.X);
  float x[kRb][kNc][8];
  Eight<T> raw[kRb][kNc];
  Eight<__bf16> o[kRb][kNc];
  EightCodes c[kRb][kNc];
#pragma unroll
  for (int r = 0; r < kRb; ++r)
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * 8;
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
      const int col = (k * blockDim.x + threadIdx.x) * 8;
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
          const int col = (k * blockDim.x + threadIdx.x) * 8;
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
    const int col = (k * blockDim.x + threadIdx.x) * 8;
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
  float* part_gate;                // [2][workgroups][d]: of the gate's row that began before the workgroup's rows; of the one that goes on behind them
  float offset, eps, scale, inv_d;
  int S, d, normalize, gate_rows;
  int rows;                        // of a workgroup
};

// dw_post and dgate of eight columns from t = sum of dY * N / w_post over the rows of a call without a gate, or whose
// rows share one gate.
__device__ __forceinline__ void finish_post(const NormBwd& a, int col, const float (&t)[8]) {
  float w[8], g[8], v[8];
  weights(a.gate, 0.f, col, true, g);
  if (a.dw_post) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a.scale * g[i] * t[i];
    Eight<float> e;
    e.set(v);
    e.store(a.dw_post + col);
  }
  if (a.dgate) {
    weights(a.normalize ? a.w_post : nullptr, a.normalize ? a.offset : 0.f, col, true, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a.scale * w[i] * t[i];
    Eight<float> e;
    e.set(v);
    e.store(a.dgate + col);
  }
}

// kMany: more than one row of gates.
template <class T, bool kPre, bool kRes, bool kMany, int kNc, int kRb>
__global__ __launch_bounds__(1024) void k_norm_bwd(const NormBwd a) {
  constexpr int kFirst = (kPre ? 2 : 0) + (kRes ? kPre ? 1 : 2 : 0);   // sums over a row that wait for nothing
  __shared__ float lds1[2][kNormMaxWaves][kFirst * kRb], lds2[2][kNormMaxWaves][kRb];
  RowSums<kFirst * kRb> first_sums(lds1);
  RowSums<kRb> second_sums(lds2);
  const int d = a.d, blocks = (d + 31) / 32;
  const int begin = blockIdx.x * a.rows, end = min(begin + a.rows, a.S);
  const bool need_o = kRes && (a.O || a.codes_o);
  float acc_pre[kNc][8] = {}, acc_post[kNc][8] = {}, acc_gate[kNc][8] = {};
  int group = kMany ? begin / a.gate_rows : 0;      // the gate's row that acc_gate belongs to
  for (int r0 = begin; r0 < end; r0 += kRb) {
    Eight<__bf16> dh[kRb][kNc], o[kRb][kNc];
    Eight<T> x[kRb][kNc], dy[kRb][kNc];
    EightCodes cx[kRb][kNc], co[kRb][kNc];
#pragma unroll
    for (int r = 0; r < kRb; ++r)
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        const int col = (k * blockDim.x + threadIdx.x) * 8;
        if (r0 + r >= end || col >= d) continue;
        const size_t at = (size_t)(r0 + r) * d + col, block = (size_t)(r0 + r) * blocks + col / 32;
        if (kPre) {
          dh[r][k].load(a.dH + at);
          if (a.codes_x) cx[r][k].load(a.codes_x + at, a.exps_x + block);
          else x[r][k].load(static_cast<const T*>(a.X) + at);
          if (a.dres) dy[r][k].load(static_cast<const T*>(a.dres) + at);
        } else {
          dy[r][k].load(static_cast<const T*>(a.dY) + at);
        }
        if (need_o) {
          if (a.codes_o) co[r][k].load(a.codes_o + at, a.exps_o + block);
          else o[r][k].load(a.O + at);
        }
      }
    auto get_x = [&](int r, int k, float (&v)[8]) { a.codes_x ? cx[r][k].get(v) : x[r][k].get(v); };
    auto get_o = [&](int r, int k, float (&v)[8]) { a.codes_o ? co[r][k].get(v) : o[r][k].get(v); };
    auto get_gate = [&](int r, int col, float (&g)[8]) {      // times the scale
      const bool on = col < d && r0 + r < end;
      weights(a.gate ? a.gate + (kMany ? (size_t)((unsigned)(r0 + r) / (unsigned)a.gate_rows) * d : 0) : nullptr, 0.f, col, on, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] *= a.scale;
    };
    float sums[kFirst * kRb];
#pragma unroll
    for (int i = 0; i < kFirst * kRb; ++i) sums[i] = 0.f;
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * 8;
      float w[8], wo[8];
      if (kPre) weights(a.w_pre, a.offset, col, col < d, w);
      if (kRes && a.normalize) weights(a.w_post, a.offset, col, col < d, wo);
#pragma unroll
      for (int r = 0; r < kRb; ++r) {
        float* const s = sums + r * kFirst;
        if (kPre) {
          float xv[8], hv[8];
          get_x(r, k, xv);
          dh[r][k].get(hv);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            s[0] = fmaf(xv[i], xv[i], s[0]);
            s[1] = fmaf(hv[i] * w[i], xv[i], s[1]);
          }
        }
        if (kRes && a.normalize) {
          float ov[8];
          get_o(r, k, ov);
          float* const so = s + (kPre ? 2 : 0);
#pragma unroll
          for (int i = 0; i < 8; ++i) so[0] = fmaf(ov[i], ov[i], so[0]);
          if (!kPre) {
            float g[8], yv[8];
            get_gate(r, col, g);
            dy[r][k].get(yv);
#pragma unroll
            for (int i = 0; i < 8; ++i) so[1] = fmaf(g[i] * yv[i] * wo[i], ov[i], so[1]);
          }
        }
      }
    }
    if (kPre || a.normalize) first_sums(sums);
    float dyv[kRb][kNc][8];
    float post[kRb];               // sum of b * O
    float rstd_o[kRb];
#pragma unroll
    for (int r = 0; r < kRb; ++r) {
      post[r] = 0.f;
      rstd_o[r] = kRes && a.normalize ? rsqrtf(fmaf(sums[r * kFirst + (kPre ? 2 : 0)], a.inv_d, a.eps)) : 1.f;
      if (!kPre) post[r] = sums[r * kFirst + (kFirst - 1)];
    }
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * 8;
      float w[8], wo[8];
      if (kPre) weights(a.w_pre, a.offset, col, col < d, w);
      if (kPre && kRes && a.normalize) weights(a.w_post, a.offset, col, col < d, wo);
#pragma unroll
      for (int r = 0; r < kRb; ++r) {
        dy[r][k].get(dyv[r][k]);
        if (!kPre) continue;
        const float rstd = rsqrtf(fmaf(sums[r * kFirst], a.inv_d, a.eps));
        const float c = sums[r * kFirst + 1] * rstd * a.inv_d;
        float xv[8], hv[8];
        get_x(r, k, xv);
        dh[r][k].get(hv);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float xh = xv[i] * rstd;
          acc_pre[k][i] = fmaf(hv[i], xh, acc_pre[k][i]);
          dyv[r][k][i] += rstd * (hv[i] * w[i] - xh * c);
        }
        if (r0 + r < end && col < d) {
          Eight<T> e;
          e.set(dyv[r][k]);
          e.store(static_cast<T*>(a.dX) + (size_t)(r0 + r) * d + col);
        }
        if (kRes && a.normalize) {
          float ov[8], g[8];
          get_o(r, k, ov);
          get_gate(r, col, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) post[r] = fmaf(g[i] * dyv[r][k][i] * wo[i], ov[i], post[r]);
        }
      }
    }
    if (!kRes) continue;
    if (kPre && a.normalize) second_sums(post);
#pragma unroll
    for (int r = 0; r < kRb; ++r) {
      const bool last = kMany && r0 + r < end && (r0 + r + 1 == end || (r0 + r + 1) % a.gate_rows == 0);
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        const int col = (k * blockDim.x + threadIdx.x) * 8;
        const bool on = col < d && r0 + r < end;
        float g[8], ov[8] = {}, out[8], wo[8];
        get_gate(r, col, g);
        if (need_o) get_o(r, k, ov);
        if (a.normalize) weights(a.w_post, a.offset, col, col < d, wo);
        const float c = post[r] * rstd_o[r] * a.inv_d;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float oh = ov[i] * rstd_o[r], e = g[i] * dyv[r][k][i];
          out[i] = a.normalize ? rstd_o[r] * (e * wo[i] - oh * c) : e;
          const float t = dyv[r][k][i] * oh;
          if (kMany) {
            acc_post[k][i] = fmaf(e, oh, acc_post[k][i]);
            acc_gate[k][i] += t;
          } else {
            acc_post[k][i] += t;
          }
        }
        if (on) {
          Eight<__bf16> e;
          e.set(out);
          e.store(a.dO + (size_t)(r0 + r) * d + col);
        }
        if (kMany && last) {
          const int64_t from = (int64_t)group * a.gate_rows, to = min(from + a.gate_rows, (int64_t)a.S);
          if (from >= begin && to <= end) {
            float wv[8];
            weights(a.normalize ? a.w_post : nullptr, a.normalize ? a.offset : 0.f, col, col < d, wv);
#pragma unroll
            for (int i = 0; i < 8; ++i) wv[i] *= a.scale * acc_gate[k][i];
            Eight<float> e;
            e.set(wv);
            if (col < d) e.store(a.dgate + (size_t)group * d + col);
          } else {
            Eight<float> e;
            e.set(acc_gate[k]);
            if (col < d) e.store(a.part_gate + ((size_t)(from < begin ? 0 : gridDim.x) + blockIdx.x) * d + col);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) acc_gate[k][i] = 0.f;
        }
      }
      if (last) ++group;
    }
  }
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    const int col = (k * blockDim.x + threadIdx.x) * 8;
    if (col >= d) continue;
    Eight<float> e;
    if (kPre && a.dw_pre) {
      e.set(acc_pre[k]);
      e.store((gridDim.x == 1 ? a.dw_pre : a.part_pre + (size_t)blockIdx.x * d) + col);
    }
    if (kRes && (a.dw_post || (a.dgate && !kMany))) {
      if (gridDim.x == 1 && !kMany) {
        finish_post(a, col, acc_post[k]);
      } else {
        e.set(acc_post[k]);
        e.store((gridDim.x == 1 ? a.dw_post : a.part_post + (size_t)blockIdx.x * d) + col);
      }
    }
  }
}

// Sums of the workgroups' sums: blockIdx.y = 0 dw_pre, 1 dw_post (and the gradient of a single row of gates), from 2 on the
// rows of the gate that lie in more than one workgroup: each row of the gate in turn where it has at least as
// many rows as a workgroup, else those across the border behind each workgroup.  A workgroup takes 64 columns: 16 lanes of
// four, and 16 groups of lanes that share out the workgroups, summed up in order.
constexpr int kReduceThreads = 256, kReduceCols = 64;
template <bool kMany>
__global__ __launch_bounds__(kReduceThreads) void k_norm_reduce(const NormBwd a, int n) {
  __shared__ norm_f32x4 lds[16][16];
  const int lane = threadIdx.x % 16, slice = threadIdx.x / 16, d = a.d;
  const int col = blockIdx.x * kReduceCols + lane * 4;
  const float* part = blockIdx.y == 0 ? a.part_pre : a.part_post;
  int first = 0, last = n - 1, group = 0;
  if (blockIdx.y == 0 ? !a.dw_pre : blockIdx.y == 1 ? !(a.dw_post || (a.dgate && !kMany)) : !kMany) return;
  if (blockIdx.y >= 2) {
    const int i = blockIdx.y - 2;
    group = a.gate_rows >= a.rows ? i : (int)(((int64_t)(i + 1) * a.rows - 1) / a.gate_rows);
    const int64_t from = (int64_t)group * a.gate_rows, to = min(from + a.gate_rows, (int64_t)a.S);
    first = (int)(from / a.rows);
    last = (int)((to - 1) / a.rows);
    if (first == last) return;               // written by the workgroup
    part = a.part_gate;
  }
  norm_f32x4 sum = {0, 0, 0, 0};
  if (col < d) {
    for (int p = first + slice; p <= last; p += 16) {
      const size_t at = (blockIdx.y >= 2 && p == first ? (size_t)n : 0) + p;
      sum += *reinterpret_cast<const norm_f32x4*>(part + at * d + col);
    }
  }
  lds[slice][lane] = sum;
  __syncthreads();
  if (slice || col >= d) return;
  for (int s = 1; s < 16; ++s) sum += lds[s][lane];
  float f[4];
  for (int i = 0; i < 4; ++i) f[i] = sum[i];
  auto weight = [&](const __bf16* w, float offset, int i) { return offset + (w ? (float)w[col + i] : 1.f); };
  auto put = [&](float* out, auto factor) {
    norm_f32x4 v;
    for (int i = 0; i < 4; ++i) v[i] = f[i] * factor(i);
    *reinterpret_cast<norm_f32x4*>(out + col) = v;
  };
  auto n_weight = [&](int i) { return a.scale * weight(a.normalize ? a.w_post : nullptr, a.normalize ? a.offset : 0.f, i); };
  if (blockIdx.y == 0) put(a.dw_pre, [](int) { return 1.f; });
  else if (blockIdx.y >= 2) put(a.dgate + (size_t)group * d, n_weight);
  else {
    if (a.dw_post) put(a.dw_post, [&](int i) { return kMany ? 1.f : a.scale * weight(a.gate, 0.f, i); });
    if (!kMany && a.dgate) put(a.dgate, n_weight);
  }
}

}  // namespace mst
