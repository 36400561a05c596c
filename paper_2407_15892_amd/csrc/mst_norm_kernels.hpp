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
  __device__ void load_streamed(const __bf16* p) { u = __builtin_nontemporal_load(reinterpret_cast<const norm_u32x4*>(p)); }
  __device__ void store_streamed(__bf16* p) const { __builtin_nontemporal_store(u, reinterpret_cast<norm_u32x4*>(p)); }
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
  __device__ void load_streamed(const float* p) { load(p); }            // halves of a line: not past the caches
  __device__ void store_streamed(float* p) const { store(p); }
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
  template <bool kStream> __device__ void load(const int8_t* codes, const uint8_t* exp) {
    const norm_u32x2* const p = reinterpret_cast<const norm_u32x2*>(codes);
    c = kStream ? __builtin_nontemporal_load(p) : *p;
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
template <class T> constexpr int kCkptEights = sizeof(T) == 2 ? 2 : 1;      // eights per lane, a workgroup's lanes apart

// One lane per eight entries; a row takes a whole number of quads, so that a quad is a block.
template <class T, bool kStream>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_pack(const T* X, FastDiv per_row, uint32_t slots, int d, int8_t* codes, uint8_t* exps) {
  constexpr int kEights = kCkptEights<T>;
  Eight<T> x[kEights];
  uint32_t n[kEights];
  size_t at[kEights];
  bool on[kEights];
#pragma unroll
  for (int i = 0; i < kEights; ++i) {
    n[i] = (blockIdx.x * kEights + i) * kCkptThreads + threadIdx.x;
    const uint32_t row = per_row(n[i] < slots ? n[i] : 0), in_row = n[i] - row * per_row.d;
    on[i] = n[i] < slots && (int)in_row * 8 < d;
    at[i] = (size_t)row * d + in_row * 8;
    if (on[i]) kStream ? x[i].load_streamed(X + at[i]) : x[i].load(X + at[i]);
  }
#pragma unroll
  for (int i = 0; i < kEights; ++i) {
    float v[8];
    x[i].get(v);
    const Packed p = pack_eight(v);
    if (!on[i]) continue;
    __builtin_nontemporal_store(p.codes, reinterpret_cast<norm_u32x2*>(codes + at[i]));
    if (threadIdx.x % 4 == 0) exps[n[i] >> 2] = (uint8_t)p.exp;
  }
}

template <class T, bool kStream>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_unpack(const int8_t* codes, const uint8_t* exps, FastDiv per_row, uint32_t slots, int d, T* X) {
  constexpr int kEights = kCkptEights<T>;
  EightCodes c[kEights];
  size_t at[kEights];
  bool on[kEights];
#pragma unroll
  for (int i = 0; i < kEights; ++i) {
    const uint32_t n = (blockIdx.x * kEights + i) * kCkptThreads + threadIdx.x;
    const uint32_t row = per_row(n < slots ? n : 0), in_row = n - row * per_row.d;
    on[i] = n < slots && (int)in_row * 8 < d;
    at[i] = (size_t)row * d + in_row * 8;
    if (on[i]) c[i].template load<kStream>(codes + at[i], exps + (n >> 2));
  }
#pragma unroll
  for (int i = 0; i < kEights; ++i) {
    if (!on[i]) continue;
    float v[8];
    c[i].get(v);
    Eight<T> x;
    x.set(v);
    x.store_streamed(X + at[i]);
  }
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

// ---- rows and weights in memory ------------------------------------------------------------------------------------------

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
constexpr int kStorePolicy = kNonTemporalAccess;

template <int kPolicy, class T> __device__ __forceinline__ void load_eight(Eight<T>& e, __amdgpu_buffer_rsrc_t rows, uint32_t at) {
  const uint32_t byte = at * (uint32_t)sizeof(T);
  if constexpr (sizeof(T) == 2) {
    e.u = __builtin_bit_cast(norm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, byte, 0, kPolicy));
  } else {
    e.a = __builtin_bit_cast(norm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, byte, 0, 0));
    e.b = __builtin_bit_cast(norm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, byte + 16, 0, 0));
  }
}
template <class T> __device__ __forceinline__ void store_eight(const Eight<T>& e, __amdgpu_buffer_rsrc_t rows, uint32_t at) {
  const uint32_t byte = at * (uint32_t)sizeof(T);
  if constexpr (sizeof(T) == 2) {
    __builtin_amdgcn_raw_buffer_store_b128(e.u, rows, byte, 0, kStorePolicy);
  } else {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(norm_u32x4, e.a), rows, byte, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(norm_u32x4, e.b), rows, byte + 16, 0, 0);
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

// Eight weights (or gates); the buffer of ones that are not there is empty.
__device__ __forceinline__ Eight<__bf16> load_weights(const __bf16* w, int d, int col) {
  Eight<__bf16> e;
  load_eight<0>(e, rows_of(w, 0, 1, 2 * d), col < d ? col : kNoColumn);
  return e;
}
__device__ __forceinline__ void weights(const Eight<__bf16>& e, bool there, float offset, float (&v)[8]) {
  e.get(v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = offset + (there ? v[i] : 1.f);
}

// ---- forward -------------------------------------------------------------------------------------------------------------

struct NormFwd {
  const void* X;                   // stream type; NULL with kRebuild, where codes_x stand for it
  const __bf16* O;
  const __bf16 *w_pre, *w_post;    // NULL: ones
  const __bf16* gate;              // NULL: ones
  void* Y;
  __bf16* H;
  const int8_t* codes_x; const uint8_t* exps_x;
  int8_t* codes_o; uint8_t* exps_o;
  int8_t* codes_y; uint8_t* exps_y;      // of Y, or without kRes of X
  float offset, eps, scale, inv_d;
  int S, d, normalize;
  int gate_rows, gates;            // without a gate S and 1
  int row0;                        // first row of the launch
  Team team;
};

__device__ __forceinline__ void store_packed(const Packed& p, __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t exps, uint32_t at, uint32_t block) {
  __builtin_amdgcn_raw_buffer_store_b64(p.codes, codes, at, 0, kStorePolicy);
  __builtin_amdgcn_raw_buffer_store_b8((unsigned char)p.exp, exps, threadIdx.x % 4 ? kNoColumn : block, 0, 0);
}

// kRb rows per team, kNc chunks of 8 columns per lane.
template <class T, bool kRes, bool kPre, bool kRebuild, int kPolicy, int kNc, int kRb>
__global__ __launch_bounds__(1024) void k_norm_fwd(const NormFwd a) {
  __shared__ float lds[2][kNormMaxWaves][kRb];
  RowSums<kRb> row_sums(lds, a.team);
  const int threads = a.team.threads(), lane = threadIdx.x % threads, teams = blockDim.x / threads, in_block = threadIdx.x / threads;
  const int d = a.d, blocks = (d + 31) / 32;
  const int first = a.row0 + (int)blockIdx.x * teams * kRb;
  const int rows = min(teams * kRb, a.S - first);        // of the workgroup
  const int first_gate = a.gates > 1 ? first / a.gate_rows : 0;
  uint32_t at[kRb][kNc], block[kRb][kNc], gate_at[kRb][kNc];
  Source<T, kRebuild, kPolicy> raw[kRb][kNc];
  Eight<__bf16> o[kRb][kNc], g[kRb][kNc], w[kNc], wo[kNc];
#pragma unroll
  for (int r = 0; r < kRb; ++r) {
    const int row = r * teams + in_block;
    const int gate = a.gates > 1 ? (first + row - first_gate * a.gate_rows) / a.gate_rows : 0;
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      const int col = (k * threads + lane) * 8;
      at[r][k] = col < d ? row * d + col : kNoColumn;
      block[r][k] = col < d ? row * blocks + col / 32 : kNoColumn;
      gate_at[r][k] = col < d ? gate * d + col : kNoColumn;
      raw[r][k].load(kRebuild ? rows_of(a.codes_x, first, rows, d) : rows_of(a.X, first, rows, (int)sizeof(T) * d), rows_of(a.exps_x, first, rows, blocks),
                     at[r][k], block[r][k]);
      if (kRes) load_eight<kPolicy>(o[r][k], rows_of(a.O, first, rows, 2 * d), at[r][k]);
    }
  }
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    const int col = (k * threads + lane) * 8;
    if (kRes) {
      wo[k] = load_weights(a.w_post, d, col);
#pragma unroll
      for (int r = 0; r < kRb; ++r) load_eight<0>(g[r][k], rows_of(a.gate, first_gate, min(teams * kRb, a.gates - first_gate), 2 * d), gate_at[r][k]);
    }
    if (kPre) w[k] = load_weights(a.w_pre, d, col);
  }
  const __amdgpu_buffer_rsrc_t codes_y = rows_of(a.codes_y, first, rows, d), exps_y = rows_of(a.exps_y, first, rows, blocks);
  float x[kRb][kNc][8];
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
      float wv[8];
      weights(wo[k], a.normalize && a.w_post, a.normalize ? a.offset : 0.f, wv);
#pragma unroll
      for (int r = 0; r < kRb; ++r) {
        float v[8], base[8], gv[8];
        o[r][k].get(v);
        if (a.codes_o)
          store_packed(pack_eight(v), rows_of(a.codes_o, first, rows, d), rows_of(a.exps_o, first, rows, blocks), at[r][k], block[r][k]);
        raw[r][k].get(base);
        weights(g[r][k], a.gate != nullptr, 0.f, gv);
        const float q = a.normalize ? rstd[r] : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[r][k][i] = fmaf(a.scale * gv[i], v[i] * q * wv[i], base[i]);
        Eight<T> y;
        y.set(x[r][k]);
        store_eight(y, rows_of(a.Y, first, rows, (int)sizeof(T) * d), at[r][k]);
        if (kPre && a.codes_y) {
          y.get(base);
          store_packed(pack_eight(base), codes_y, exps_y, at[r][k], block[r][k]);
        }
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < kRb; ++r)
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        raw[r][k].get(x[r][k]);
        if (!kRebuild && a.codes_y) store_packed(pack_eight(x[r][k]), codes_y, exps_y, at[r][k], block[r][k]);
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
  for (int k = 0; k < kNc; ++k) {
    float wv[8];
    weights(w[k], a.w_pre != nullptr, a.offset, wv);
#pragma unroll
    for (int r = 0; r < kRb; ++r) {
      const float q = rsqrtf(fmaf(rstd[r], a.inv_d, a.eps));
      float h[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = x[r][k][i] * q * wv[i];
      Eight<__bf16> e;
      e.set(h);
      store_eight(e, rows_of(a.H, first, rows, 2 * d), at[r][k]);
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
  int gate_rows, gates;            // without a gate S and 1
  int share;                       // workgroups that share a row of the gate (not kWhole)
  int rows;                        // that a team takes in turn
  Team team;
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
  // The gate's rows of the workgroup's teams.
  auto load_gate = [&](int k) {
    Eight<__bf16> g;
    load_eight<0>(g, rows_of(a.gate, group, max(0, min(kWhole ? teams : 1, a.gates - group)), 2 * d), column(k) < d ? (kWhole ? in_block * d : 0) + column(k) : kNoColumn);
    return g;
  };
  auto set_f = [&](int k, const Eight<__bf16>& gate, const Eight<__bf16>& weight) {
    float wo[8];
    weights(gate, a.gate != nullptr, 0.f, f[k]);
    weights(weight, a.normalize && a.w_post, a.normalize ? a.offset : 0.f, wo);
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
  }
#pragma unroll
  for (int slot = 0; slot < kAhead; ++slot) load(slot);
  Eight<__bf16> w_raw[kNc], wo_raw[kNc], g_raw[kNc];
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    if (kPre) w_raw[k] = load_weights(a.w_pre, d, column(k));
    if (kRes) wo_raw[k] = load_weights(a.w_post, d, column(k));
    if (kRes && !kWhole) g_raw[k] = load_gate(k);
  }
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    if (kPre) weights(w_raw[k], a.w_pre != nullptr, a.offset, w[k]);
    if (kRes && !kWhole) set_f(k, g_raw[k], wo_raw[k]);
  }
  auto one_row = [&](int slot) {
    float dh[kNc][8], x[kNc][8], dy[kNc][8], o[kNc][8];
    float sums[kFirst];
#pragma unroll
    for (int i = 0; i < kFirst; ++i) sums[i] = 0.f;
    if (kWhole && in_group == 0) {
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        g_raw[k] = load_gate(k);
        set_f(k, g_raw[k], wo_raw[k]);
      }
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
      const float q = rsqrtf(fmaf(sums[0], a.inv_d, a.eps)), c = -(sums[1] * a.inv_d * q) * q * q;      // q^3 alone leaves the range
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
      const float c = a.normalize ? -(post[0] * a.inv_d * q) * q * q : 0.f;
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
          float v[8], gv[8];
          weights(wo_raw[k], a.normalize && a.w_post, a.normalize ? a.offset : 0.f, v);
          weights(g_raw[k], true, 0.f, gv);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            acc_post[k][i] = fmaf(a.scale * gv[i], acc_group[k][i], acc_post[k][i]);
            v[i] *= a.scale * acc_group[k][i];
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
  // As many rows in every team, for the barriers; zeros behind the last one.
  int i_row = 0;
  for (; i_row + kAhead <= a.rows; i_row += kAhead) {
#pragma unroll
    for (int slot = 0; slot < kAhead; ++slot) one_row(slot);
  }
  if (kAhead > 1 && i_row < a.rows) one_row(0);
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
#pragma unroll 4
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

// Four weights as floats, ones where there are none.
struct Four {
  norm_f32x4 v;
  __device__ void load(const __bf16* w, size_t at, float offset) {
    norm_u32x2 u = {0x3f803f80u, 0x3f803f80u};
    if (w) u = *reinterpret_cast<const norm_u32x2*>(w + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = offset + __uint_as_float(i % 2 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
  }
};

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
  // what the sums are multiplied with, loaded beside them
  const bool on = col < d;
  Four w, g;
  w.load(a.normalize ? a.w_post : nullptr, on ? col : 0, a.normalize ? a.offset : 0.f);
  g.load(a.gate, (size_t)(blockIdx.y >= 2 ? min(group, gates - 1) : 0) * d + (on ? col : 0), 0.f);
  norm_f32x4 sum = {0, 0, 0, 0};
  if (on) {
#pragma unroll 4
    for (int p = slice % slices; p < count; p += slices) {
      norm_f32x4 v = *reinterpret_cast<const norm_f32x4*>(part + (size_t)(first + p) * d + col);
      if (weighted) {
        Four of;
        of.load(a.gate, (size_t)((unsigned)p / (unsigned)a.share) * d + col, 0.f);
        v *= of.v * a.scale;
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
  if (slice % slices || !on || count == 0) return;
  auto put = [&](float* to, norm_f32x4 v) { *reinterpret_cast<norm_f32x4*>(to + col) = v; };
  if (blockIdx.y == 0) put(a.dw_pre, sum);
  else if (blockIdx.y >= 2) put(a.dgate + (size_t)group * d, sum * w.v * a.scale);
  else if (whole || weighted) put(a.dw_post, sum);
  else {
    if (a.dw_post) put(a.dw_post, sum * g.v * a.scale);
    if (one_gate) put(a.dgate, sum * w.v * a.scale);
  }
}

}  // namespace mst
