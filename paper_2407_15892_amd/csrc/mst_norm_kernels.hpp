// Device kernels between the mini-sequence blocks (gfx950): norms, the gated residual, their gradients, and 8-bit
// checkpoints.  The formulas are in include/mst_norm.h.
//
//   k_ckpt_pack, k_ckpt_unpack   the checkpoint alone
//   k_norm_fwd                   norm before a block, residual after it, or both
//   k_norm_bwd                   their gradients; per workgroup sums over its rows for those of weights and gates
//   k_norm_reduce                these sums over the workgroups, in fixed order
//
// All of them move data and compute little, so a row is read once: a team of lanes holds it in registers, sums over the row go
// through DPP and LDS, and what is needed of the row is written from the registers.  A lane has eight columns of each chunk of
// the row: adjacent ones (16 bytes of bf16) with a bf16 stream, twice four half a chunk apart with a float32 one, so that a
// wave's access to its 16 bytes per lane is whole cache lines either way (float32 unpack of 8192 x 4096, half lines 34.6 us, whole
// ones 24.8).  Four or eight adjacent lanes hold the 32 columns of a checkpoint's block.
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

// Eight entries of a checkpoint, each four of them with the exponent of their block.
struct EightCodes {
  unsigned c[2] = {0, 0}, e[2] = {0, 0};
  __device__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // 2^(e - 127): of 0 a subnormal, of 255 NaN
      const float scale = __uint_as_float(max(e[i] << 23 | ((e[i] + 1) >> 8) << 22, 0x00400000u));
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

// Codes of kN entries and the exponent byte of their block of 32, whose other entries are in the 32 / kN lanes around (all of
// them call this; lanes behind the row's end hold zeros).  The least scale whose product with 127.5 is more than
// the largest magnitude m * 2^e: 2^(e - 6), or 2^(e - 5) from m = 127.5 / 64 = 1 + 127 / 128 on, where adding the last bit of
// that mantissa carries into the exponent.  x / scale + 1.5 * 2^23 rounds to the nearest integer, ties to even, and has its
// two's complement in the low byte.  Measured as integers magnitudes order NaN above infinity above all else.
template <int kN> struct Packed { unsigned codes[kN / 4], exp; };
template <int kN> __device__ __forceinline__ Packed<kN> pack(const float* v) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < kN; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max(top, dpp_u32<kQuadSwap1>(top));
  top = max(top, dpp_u32<kQuadSwap2>(top));
  if (kN == 4) top = max(top, dpp_u32<kHalfMirror>(top));
  const unsigned E = (top + 0x10000u) >> 23;
  Packed<kN> p;
  p.exp = E >= 255 ? 255 : max(E, 6u) - 6;
  const float inverse = __uint_as_float((254u - p.exp) << 23);
  unsigned b[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) b[i] = __float_as_uint(fmaf(v[i], inverse, 12582912.f));
#pragma unroll
  for (int i = 0; i < kN / 4; ++i)      // the low bytes of four words
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
constexpr int kCkptParts = 2;                                          // parts of 16 bytes per lane, a workgroup's lanes apart
template <class T> constexpr int kCkptPart = 16 / sizeof(T);           // entries of one

// 131072 x 4096 bf16: 249 us to pack, 247 to unpack (6.5 and 6.6 TB/s).
// One lane per part; a row takes a whole number of blocks, whose 32 entries are in adjacent lanes.
template <class T, bool kStream>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_pack(const T* X, FastDiv per_row, uint32_t parts, int d, int8_t* codes, uint8_t* exps) {
  constexpr int kN = kCkptPart<T>;
  norm_u32x4 x[kCkptParts];
  uint32_t n[kCkptParts];
  size_t at[kCkptParts];
  bool on[kCkptParts];
#pragma unroll
  for (int i = 0; i < kCkptParts; ++i) {
    n[i] = (blockIdx.x * kCkptParts + i) * kCkptThreads + threadIdx.x;
    const uint32_t row = per_row(n[i] < parts ? n[i] : 0), in_row = n[i] - row * per_row.d;
    on[i] = n[i] < parts && (int)in_row * kN < d;
    at[i] = (size_t)row * d + in_row * kN;
    const norm_u32x4* const p = reinterpret_cast<const norm_u32x4*>(X + at[i]);
    x[i] = norm_u32x4{0, 0, 0, 0};
    if (on[i]) x[i] = kStream ? __builtin_nontemporal_load(p) : *p;
  }
#pragma unroll
  for (int i = 0; i < kCkptParts; ++i) {
    float v[kN];
    if constexpr (kN == 8) {
      Eight<__bf16> e;
      e.u = x[i];
      e.get(v);
    } else {
      for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(x[i][k]);
    }
    const Packed<kN> p = pack<kN>(v);
    if (!on[i]) continue;
    if constexpr (kN == 8) __builtin_nontemporal_store(norm_u32x2{p.codes[0], p.codes[1]}, reinterpret_cast<norm_u32x2*>(codes + at[i]));
    else __builtin_nontemporal_store(p.codes[0], reinterpret_cast<unsigned*>(codes + at[i]));
    if (threadIdx.x % (32 / kN) == 0) exps[n[i] / (32 / kN)] = (uint8_t)p.exp;
  }
}

template <class T, bool kStream>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_unpack(const int8_t* codes, const uint8_t* exps, FastDiv per_row, uint32_t parts, int d,
                                                             T* X) {
  constexpr int kN = kCkptPart<T>;
  EightCodes c[kCkptParts];
  size_t at[kCkptParts];
  bool on[kCkptParts];
#pragma unroll
  for (int i = 0; i < kCkptParts; ++i) {
    const uint32_t n = (blockIdx.x * kCkptParts + i) * kCkptThreads + threadIdx.x;
    const uint32_t row = per_row(n < parts ? n : 0), in_row = n - row * per_row.d;
    on[i] = n < parts && (int)in_row * kN < d;
    at[i] = (size_t)row * d + in_row * kN;
    if (!on[i]) continue;
    const unsigned* const p = reinterpret_cast<const unsigned*>(codes + at[i]);
    if constexpr (kN == 8) {
      const norm_u32x2* const q = reinterpret_cast<const norm_u32x2*>(p);
      const norm_u32x2 u = kStream ? __builtin_nontemporal_load(q) : *q;
      c[i].c[0] = u[0];
      c[i].c[1] = u[1];
    } else {
      c[i].c[0] = kStream ? __builtin_nontemporal_load(p) : *p;
    }
    c[i].e[0] = c[i].e[1] = exps[n / (32 / kN)];
  }
#pragma unroll
  for (int i = 0; i < kCkptParts; ++i) {
    if (!on[i]) continue;
    float v[8];
    c[i].get(v);
    norm_u32x4 x;
    if constexpr (kN == 8) {
      Eight<__bf16> e;
      e.set(v);
      x = e.u;
    } else {
      for (int k = 0; k < 4; ++k) x[k] = __float_as_uint(v[k]);
    }
    __builtin_nontemporal_store(x, reinterpret_cast<norm_u32x4*>(X + at[i]));
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
    if (__builtin_expect(team.lanes < 64, 0)) {
      if (team.lanes == 8) return;
      add_dpp<kMirror>(v);
      if (team.lanes == 16) return;
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v[i]), 0x401f));   // lane ^ 16
      return;
    }
    add_dpp<kMirror>(v);
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
// Rows whose loads are under way while one is summed up.  Norm's backward of 32768 x 4096, bf16: one 160 us, two 155; of float32 (73, 75 of
// 8192 x 4096) and of the others, which load more or have fewer registers left, two are slower.
template <class T> constexpr int rows_ahead(bool pre, bool res, int chunks) { return pre && !res && chunks == 1 && sizeof(T) == 2 ? 2 : 1; }

constexpr int kNonTemporalAccess = 2;         // cache policy of buffer loads and stores
// Results are written past the caches, which keep what comes in: 8192 x 4096, norm with checkpoint 33.4 us -> 29.7.  What reads them much later, as a
// backward pass does, loses nothing; a pass right behind this one reads from memory what the caches might have held.  The norm with checkpoint and the
// MLP's forward on its H, in a captured graph, us, past the caches and through them: d = 4096, I = 14336: 1 and 64 rows the same, 512 rows 222, 215, 2048 rows
// 568, 566, 8192 rows 2072, 2067; d = 1024, I = 2816: 1 and 64 rows the same, 512 rows 30.0, 27.1, 2048 rows 63.4, 60.3, 8192 rows 242, 229.
constexpr int kStorePolicy = kNonTemporalAccess;

// A lane's columns: entries 0..3 from column a on, entries 4..7 from b (kApart: half a chunk apart; else b = a + 4, and the access is
// one of eight entries).  Also offsets of these entries, and of their blocks' exponents.
struct Pair { uint32_t a, b; };
template <bool kApart> __device__ __forceinline__ Pair columns(int chunk, int threads, int lane, int d) {
  const uint32_t a = kApart ? (2 * chunk * threads + lane) * 4 : (chunk * threads + lane) * 8, b = a + (kApart ? 4 * threads : 4);
  return {a < (uint32_t)d ? a : kNoColumn, b < (uint32_t)d ? b : kNoColumn};
}
__device__ __forceinline__ Pair in_row(Pair columns, uint32_t row_at) {
  return {columns.a == kNoColumn ? kNoColumn : row_at + columns.a, columns.b == kNoColumn ? kNoColumn : row_at + columns.b};
}
__device__ __forceinline__ Pair blocks_in_row(Pair columns, uint32_t row_at) {
  return {columns.a == kNoColumn ? kNoColumn : row_at + columns.a / 32, columns.b == kNoColumn ? kNoColumn : row_at + columns.b / 32};
}

template <bool kApart, int kPolicy, class T> __device__ __forceinline__ void load_eight(Eight<T>& e, __amdgpu_buffer_rsrc_t rows, Pair at) {
  if constexpr (sizeof(T) == 4) {
    e.a = __builtin_bit_cast(norm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at.a * 4, 0, kPolicy));
    e.b = __builtin_bit_cast(norm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at.b * 4, 0, kPolicy));
  } else if constexpr (kApart) {
    const norm_u32x2 a = __builtin_bit_cast(norm_u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows, at.a * 2, 0, kPolicy));
    const norm_u32x2 b = __builtin_bit_cast(norm_u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows, at.b * 2, 0, kPolicy));
    e.u = norm_u32x4{a[0], a[1], b[0], b[1]};
  } else {
    e.u = __builtin_bit_cast(norm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at.a * 2, 0, kPolicy));
  }
}
template <bool kApart, class T> __device__ __forceinline__ void store_eight(const Eight<T>& e, __amdgpu_buffer_rsrc_t rows, Pair at) {
  if constexpr (sizeof(T) == 4) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(norm_u32x4, e.a), rows, at.a * 4, 0, kStorePolicy);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(norm_u32x4, e.b), rows, at.b * 4, 0, kStorePolicy);
  } else if constexpr (kApart) {
    __builtin_amdgcn_raw_buffer_store_b64(norm_u32x2{e.u[0], e.u[1]}, rows, at.a * 2, 0, kStorePolicy);
    __builtin_amdgcn_raw_buffer_store_b64(norm_u32x2{e.u[2], e.u[3]}, rows, at.b * 2, 0, kStorePolicy);
  } else {
    __builtin_amdgcn_raw_buffer_store_b128(e.u, rows, at.a * 2, 0, kStorePolicy);
  }
}

// A row's eight entries: the tensor's, or those of its checkpoint.
template <class T, bool kCheckpoint, bool kApart, int kPolicy> struct Source {
  Eight<T> e;
  __device__ void load(__amdgpu_buffer_rsrc_t rows, __amdgpu_buffer_rsrc_t, Pair at, Pair) { load_eight<kApart, kPolicy>(e, rows, at); }
  __device__ void get(float (&v)[8]) const { e.get(v); }
};
template <class T, bool kApart, int kPolicy> struct Source<T, true, kApart, kPolicy> {
  EightCodes e;
  __device__ void load(__amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t exps, Pair at, Pair block) {
    if constexpr (kApart) {
      e.c[0] = __builtin_amdgcn_raw_buffer_load_b32(codes, at.a, 0, kPolicy);
      e.c[1] = __builtin_amdgcn_raw_buffer_load_b32(codes, at.b, 0, kPolicy);
      e.e[0] = __builtin_amdgcn_raw_buffer_load_b8(exps, block.a, 0, kPolicy);
      e.e[1] = __builtin_amdgcn_raw_buffer_load_b8(exps, block.b, 0, kPolicy);
    } else {
      const norm_u32x2 u = __builtin_bit_cast(norm_u32x2, __builtin_amdgcn_raw_buffer_load_b64(codes, at.a, 0, kPolicy));
      e.c[0] = u[0];
      e.c[1] = u[1];
      e.e[0] = e.e[1] = __builtin_amdgcn_raw_buffer_load_b8(exps, block.a, 0, kPolicy);
    }
  }
  __device__ void get(float (&v)[8]) const { e.get(v); }
};

// The checkpoint of eight entries.
template <bool kApart>
__device__ __forceinline__ void store_checkpoint(const float (&v)[8], __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t exps, Pair at,
                                                 Pair block) {
  if constexpr (kApart) {
    const Packed<4> a = pack<4>(v), b = pack<4>(v + 4);
    __builtin_amdgcn_raw_buffer_store_b32(a.codes[0], codes, at.a, 0, kStorePolicy);
    __builtin_amdgcn_raw_buffer_store_b32(b.codes[0], codes, at.b, 0, kStorePolicy);
    __builtin_amdgcn_raw_buffer_store_b8((unsigned char)a.exp, exps, threadIdx.x % 8 ? kNoColumn : block.a, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b8((unsigned char)b.exp, exps, threadIdx.x % 8 ? kNoColumn : block.b, 0, 0);
  } else {
    const Packed<8> p = pack<8>(v);
    __builtin_amdgcn_raw_buffer_store_b64(norm_u32x2{p.codes[0], p.codes[1]}, codes, at.a, 0, kStorePolicy);
    __builtin_amdgcn_raw_buffer_store_b8((unsigned char)p.exp, exps, threadIdx.x % 4 ? kNoColumn : block.a, 0, 0);
  }
}

// Registers whose contents the compiler takes for new ones: what was derived from them before is derived again, not kept.
__device__ __forceinline__ void renew(Eight<__bf16>& e) { asm volatile("" : "+v"(e.u)); }
__device__ __forceinline__ void renew(Eight<float>& e) { asm volatile("" : "+v"(e.a), "+v"(e.b)); }
__device__ __forceinline__ void renew(EightCodes& e) { asm volatile("" : "+v"(e.c[0]), "+v"(e.c[1]), "+v"(e.e[0]), "+v"(e.e[1])); }

// Eight weights (or gates); the buffer of ones that are not there is empty.
template <bool kApart> __device__ __forceinline__ Eight<__bf16> load_weights(const __bf16* w, int d, Pair columns) {
  Eight<__bf16> e;
  load_eight<kApart, 0>(e, rows_of(w, 0, 1, 2 * d), columns);
  return e;
}
__device__ __forceinline__ void weights(const Eight<__bf16>& e, bool there, float offset, float (&v)[8]) {
  e.get(v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = offset + (there ? v[i] : 1.f);
}
// Eight sums to a row of float32.
__device__ __forceinline__ void store_sums(const float* v, float* to, Pair columns) {
  if (columns.a != kNoColumn) *reinterpret_cast<norm_f32x4*>(to + columns.a) = norm_f32x4{v[0], v[1], v[2], v[3]};
  if (columns.b != kNoColumn) *reinterpret_cast<norm_f32x4*>(to + columns.b) = norm_f32x4{v[4], v[5], v[6], v[7]};
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

// kRb rows per team, kNc chunks of 8 columns per lane.  Bound by memory: 32768 x 4096 bf16, norm with checkpoint 112 us (6.0 TB/s), both norms
// and checkpoints 222 (6.1).  The weights' loads follow the rows' at once: 200 x 4096, both norms, 5.8 us -> 4.2.
template <class T, bool kRes, bool kPre, bool kRebuild, int kPolicy, int kNc, int kRb>
__global__ __launch_bounds__(1024) void k_norm_fwd(const NormFwd a) {
  __shared__ float lds[2][kNormMaxWaves][kRb];
  constexpr bool kApart = sizeof(T) == 4;
  RowSums<kRb> row_sums(lds, a.team);
  const int threads = a.team.threads(), lane = threadIdx.x % threads, teams = blockDim.x / threads, in_block = threadIdx.x / threads;
  const int d = a.d, blocks = (d + 31) / 32;
  const int first = a.row0 + (int)blockIdx.x * teams * kRb;
  const int rows = min(teams * kRb, a.S - first);        // of the workgroup
  const int first_gate = a.gates > 1 ? first / a.gate_rows : 0;
  Pair at[kRb][kNc], block[kRb][kNc], gate_at[kRb][kNc];
  Source<T, kRebuild, kApart, kPolicy> raw[kRb][kNc];
  Eight<__bf16> o[kRb][kNc], g[kRb][kNc], w[kNc], wo[kNc];
#pragma unroll
  for (int r = 0; r < kRb; ++r) {
    const int row = r * teams + in_block;
    const int gate = a.gates > 1 ? (first + row - first_gate * a.gate_rows) / a.gate_rows : 0;
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      const Pair col = columns<kApart>(k, threads, lane, d);
      at[r][k] = in_row(col, row * d);
      block[r][k] = blocks_in_row(col, row * blocks);
      gate_at[r][k] = in_row(col, gate * d);
      raw[r][k].load(kRebuild ? rows_of(a.codes_x, first, rows, d) : rows_of(a.X, first, rows, (int)sizeof(T) * d),
                     rows_of(a.exps_x, first, rows, blocks), at[r][k], block[r][k]);
      if (kRes) load_eight<kApart, kPolicy>(o[r][k], rows_of(a.O, first, rows, 2 * d), at[r][k]);
    }
  }
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    const Pair col = columns<kApart>(k, threads, lane, d);
    if (kRes) {
      wo[k] = load_weights<kApart>(a.w_post, d, col);
#pragma unroll
      for (int r = 0; r < kRb; ++r)
        load_eight<kApart, 0>(g[r][k], rows_of(a.gate, first_gate, min(teams * kRb, a.gates - first_gate), 2 * d), gate_at[r][k]);
    }
    if (kPre) w[k] = load_weights<kApart>(a.w_pre, d, col);
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
          store_checkpoint<kApart>(v, rows_of(a.codes_o, first, rows, d), rows_of(a.exps_o, first, rows, blocks), at[r][k], block[r][k]);
        raw[r][k].get(base);
        weights(g[r][k], a.gate != nullptr, 0.f, gv);
        const float q = a.normalize ? rstd[r] : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[r][k][i] = fmaf(a.scale * gv[i], v[i] * q * wv[i], base[i]);
        Eight<T> y;
        y.set(x[r][k]);
        store_eight<kApart>(y, rows_of(a.Y, first, rows, (int)sizeof(T) * d), at[r][k]);
        if (kPre && a.codes_y) {
          y.get(base);
          store_checkpoint<kApart>(base, codes_y, exps_y, at[r][k], block[r][k]);
        }
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < kRb; ++r)
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        raw[r][k].get(x[r][k]);
        if (!kRebuild && a.codes_y) store_checkpoint<kApart>(x[r][k], codes_y, exps_y, at[r][k], block[r][k]);
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
      store_eight<kApart>(e, rows_of(a.H, first, rows, 2 * d), at[r][k]);
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

// Bound by memory where rows are many (32768 x 4096 bf16 from checkpoints: norm 155 us, 6.1 TB/s, residual 119, 5.7, both 238, 5.7, half of the
// vector units' time used), by latency where they are few (a row takes 2 us from its loads to its last store).
// A team takes `rows` rows in turn, the next one's loads on their way while it computes; its lanes keep the sums over them
// for their columns.  Of long rows (two chunks, d > 8192) with two norms or in float32 only what was loaded stays in registers, and
// is converted for each use (kLean): with 16 waves a lane has 128 of them, and what does not fit goes to scratch memory all the same
// (both norms: bf16 54 to 59 registers of a lane, with whole rows of the gate 94 to 102, float32 62 to 78 and 109 to 121; residual alone with
// whole rows of the gate 3 to 33).  2048 x 12288, both norms: 169 us -> 121, float32 and gated 267 -> 152, its norm alone 78 -> 60;
// bf16's norm alone 42 -> 45, and the residual's 31 -> 38, do not.
//   kWhole = false  `share` workgroups have the rows of one row of the gate (all rows without a gate), adjacent rows in
//                   adjacent teams: memory is passed through in a few streams.  Sums of dY * N, without the gate, to the workspace.
//   kWhole = true   for many short rows of gates: a team has all rows of one, then those of another; it writes their gradient
//                   and sums up dw_post.
// With x the row of X, q its rstd, a = dH * ~w: the gradient is dres + q a - x q^3 sum(a x) / d; likewise for O with
// b = dY * f, f = scale * gate * ~w_post.  One sum over the row waits for another where both norms are there.
template <class T, bool kPre, bool kRes, bool kWhole, bool kCkptX, bool kCkptO, int kPolicy, int kNc>
__global__ __launch_bounds__(1024) void k_norm_bwd(const NormBwd a) {
  constexpr int kFirst = (kPre ? 2 : 0) + (kRes ? kPre ? 1 : 2 : 0);   // sums over a row that wait for nothing
  constexpr bool kApart = sizeof(T) == 4, kLean = kNc > 1 && kPre && (kRes || kApart);
  __shared__ float lds1[2][kNormMaxWaves][kFirst], lds2[2][kNormMaxWaves][1];
  extern __shared__ norm_f32x4 lds_columns[];
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
  Pair col[kNc], at[kNc], block[kNc];
  // The gate's rows of the workgroup's teams.
  auto load_gate = [&](int k) {
    Eight<__bf16> g;
    load_eight<kApart, 0>(g, rows_of(a.gate, group, max(0, min(kWhole ? teams : 1, a.gates - group)), 2 * d),
                          in_row(col[k], kWhole ? in_block * d : 0));
    return g;
  };
  auto set_f = [&](int k, const Eight<__bf16>& gate, const Eight<__bf16>& weight) {
    float wo[8];
    weights(gate, a.gate != nullptr, 0.f, f[k]);
    weights(weight, a.normalize && a.w_post, a.normalize ? a.offset : 0.f, wo);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[k][i] *= a.scale * wo[i];
  };
  constexpr int kAhead = rows_ahead<T>(kPre, kRes, kNc);
  Eight<__bf16> dh_next[kAhead][kNc];
  Source<T, kCkptX, kApart, kPolicy> x_next[kAhead][kNc];
  Eight<T> dy_next[kAhead][kNc];
  Source<__bf16, kCkptO, kApart, kPolicy> o_next[kAhead][kNc];
  auto rows_at = [&](int64_t r) { return (int)max((int64_t)0, min((int64_t)(teams - 1) * apart + 1, end - r)); };
  auto load = [&](int slot) {
    const int rows = rows_at(next);
    const __amdgpu_buffer_rsrc_t dy_rows = rows_of(kPre ? a.dres : a.dY, next, rows, (int)sizeof(T) * d);
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      if (kPre) {
        load_eight<kApart, kPolicy>(dh_next[slot][k], rows_of(a.dH, next, rows, 2 * d), at[k]);
        x_next[slot][k].load(kCkptX ? rows_of(a.codes_x, next, rows, d) : rows_of(a.X, next, rows, (int)sizeof(T) * d),
                       rows_of(a.exps_x, next, rows, blocks), at[k], block[k]);
      }
      load_eight<kApart, kPolicy>(dy_next[slot][k], dy_rows, at[k]);
      if (kRes)
        o_next[slot][k].load(kCkptO ? rows_of(a.codes_o, next, rows, d) : rows_of(a.O, next, rows, 2 * d), rows_of(a.exps_o, next, rows, blocks),
                       at[k], block[k]);
    }
    advance(next, next_in_group);
  };
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    col[k] = columns<kApart>(k, threads, lane, d);
    at[k] = in_row(col[k], in_block * apart * d);
    block[k] = blocks_in_row(col[k], in_block * apart * blocks);
  }
  if (!kLean) {
#pragma unroll
    for (int slot = 0; slot < kAhead; ++slot) load(slot);
  }
  Eight<__bf16> w_raw[kNc], wo_raw[kNc], g_raw[kNc];
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    if (kPre) w_raw[k] = load_weights<kApart>(a.w_pre, d, col[k]);
    if (kRes && !kWhole) {
      wo_raw[k] = load_weights<kApart>(a.w_post, d, col[k]);
      g_raw[k] = load_gate(k);
    }
  }
#pragma unroll
  for (int k = 0; k < kNc; ++k) {
    if (kPre && !kLean) weights(w_raw[k], a.w_pre != nullptr, a.offset, w[k]);
    if (kRes && !kWhole && !kLean) set_f(k, g_raw[k], wo_raw[k]);
  }
  auto again_w = [&](int k) {                 // kLean: before each use
    if (!kLean) return;
    renew(w_raw[k]);
    weights(w_raw[k], a.w_pre != nullptr, a.offset, w[k]);
  };
  auto again_f = [&](int k) {
    if (!kLean) return;
    renew(g_raw[k]);
    renew(wo_raw[k]);
    set_f(k, g_raw[k], wo_raw[k]);
  };
  auto one_row = [&](int slot) {
    float dh[kNc][8], x[kNc][8], dy[kNc][8], o[kNc][8];
    float sums[kFirst];
#pragma unroll
    for (int i = 0; i < kFirst; ++i) sums[i] = 0.f;
    if (kLean) load(slot);
    if (kWhole && in_group == 0) {
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        g_raw[k] = load_gate(k);
        wo_raw[k] = load_weights<kApart>(a.w_post, d, col[k]);
        if (!kLean) set_f(k, g_raw[k], wo_raw[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kNc; ++k) {
      if (kLean) __builtin_amdgcn_sched_barrier(0);
      dy_next[slot][k].get(dy[k]);
      if (kPre) {
        again_w(k);
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
    if (!kLean) load(slot);
    const int rows = rows_at(row);
    if (kPre || a.normalize) first_sums(sums);
    float post[1] = {kPre ? 0.f : sums[1]};      // sum of b * O
    if (kPre) {
      const float q = rsqrtf(fmaf(sums[0], a.inv_d, a.eps)), c = -(sums[1] * a.inv_d * q) * q * q;      // q^3 alone leaves the range
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        if (kLean) {
          __builtin_amdgcn_sched_barrier(0);          // one chunk after the other
          renew(dy_next[slot][k]);
          renew(x_next[slot][k].e);
          renew(dh_next[slot][k]);
          dy_next[slot][k].get(dy[k]);
          x_next[slot][k].get(x[k]);
          dh_next[slot][k].get(dh[k]);
          again_w(k);
        }
        if (kLean && kRes) {
          renew(o_next[slot][k].e);
          o_next[slot][k].get(o[k]);
          again_f(k);
        }
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
        store_eight<kApart>(e, rows_of(a.dX, row, rows, (int)sizeof(T) * d), at[k]);
      }
    }
    if (kRes) {
      if (kPre && a.normalize) second_sum(post);
      const float q = a.normalize ? rsqrtf(fmaf(sums[kPre ? 2 : 0], a.inv_d, a.eps)) : 1.f;
      const float c = a.normalize ? -(post[0] * a.inv_d * q) * q * q : 0.f;
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        if (kLean) {
          __builtin_amdgcn_sched_barrier(0);
          renew(o_next[slot][k].e);
          o_next[slot][k].get(o[k]);
          again_f(k);
        }
        float out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = dy[k][i] * q;
          out[i] = u * f[k][i];
          acc_group[k][i] = fmaf(u, o[k][i], acc_group[k][i]);
        }
        if (a.normalize) {              // without the norm dO does not depend on O: 0 times an infinity or a NaN is a NaN
#pragma unroll
          for (int i = 0; i < 8; ++i) out[i] = fmaf(o[k][i], c, out[i]);
        }
        Eight<__bf16> e;
        e.set(out);
        store_eight<kApart>(e, rows_of(a.dO, row, rows, 2 * d), at[k]);
      }
      const int64_t mine = row + (int64_t)in_block * apart;
      if (kWhole && (in_group == a.gate_rows - 1 || mine == end - 1) && mine < end) {      // the last row of its row of the gate
#pragma unroll
        for (int k = 0; k < kNc; ++k) {
          float v[8], gv[8];
          // again: registers are short
          weights(load_weights<kApart>(a.w_post, d, col[k]), a.normalize && a.w_post, a.normalize ? a.offset : 0.f, v);
          weights(load_gate(k), true, 0.f, gv);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            acc_post[k][i] = fmaf(a.scale * gv[i], acc_group[k][i], acc_post[k][i]);
            v[i] *= a.scale * acc_group[k][i];
            acc_group[k][i] = 0.f;
          }
          store_sums(v, a.dgate + (size_t)(group + in_block) * d, col[k]);
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
  // the teams' sums, then to the workspace, or where they belong if this is the only workgroup: each times factor(column)
  auto put_sums = [&](const float (&acc)[kNc][8], float* to, auto factor) {
    if (teams == 1) {
#pragma unroll
      for (int k = 0; k < kNc; ++k) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t c = (i < 4 ? col[k].a : col[k].b) + i % 4;
          v[i] = acc[k][i] * (c < (uint32_t)d ? factor(c) : 0.f);
        }
        store_sums(v, to, col[k]);
      }
      return;
    }
    __syncthreads();
    if (col[0].a != kNoColumn) lds_columns[(in_block * d + col[0].a) / 4] = norm_f32x4{acc[0][0], acc[0][1], acc[0][2], acc[0][3]};
    if (col[0].b != kNoColumn) lds_columns[(in_block * d + col[0].b) / 4] = norm_f32x4{acc[0][4], acc[0][5], acc[0][6], acc[0][7]};
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
      float sum = 0.f;
#pragma unroll 4
      for (int t = 0; t < teams; ++t) sum += lds_columns[(t * d + c) / 4][c % 4];
      to[c] = sum * factor(c);
    }
  };
  const bool alone = gridDim.x == 1;
  auto one = [](int) { return 1.f; };
  auto gate_factor = [&](int c) { return a.scale * (a.gate ? (float)a.gate[c] : 1.f); };
  auto post_factor = [&](int c) { return a.scale * (a.normalize ? a.offset + (a.w_post ? (float)a.w_post[c] : 1.f) : 1.f); };
  if (kPre && a.dw_pre) put_sums(acc_pre, alone ? a.dw_pre : a.part_pre + (size_t)blockIdx.x * d, one);
  if (kRes && kWhole && a.dw_post) put_sums(acc_post, alone ? a.dw_post : a.part_post + (size_t)blockIdx.x * d, one);
  if (kRes && !kWhole && (a.dw_post || a.dgate)) {
    if (!alone) put_sums(acc_group, a.part_post + (size_t)blockIdx.x * d, one);
    else {
      if (a.dw_post) put_sums(acc_group, a.dw_post, gate_factor);
      if (a.dgate) put_sums(acc_group, a.dgate, post_factor);
    }
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
// (a power of two) share out the sums of a result, and are added up in one order.  512 sums of 4096
// columns: 4.2 us, 2 of them a launch's; with 8 rows of the gate, whose sums the workgroups of dw_post and those of dgate each read, 8.2.
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
