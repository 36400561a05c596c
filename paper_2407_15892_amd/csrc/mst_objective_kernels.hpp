// Device code of the LM head's other objectives (mst_objective.h): cross-entropy of capped logits with token weights, and
// distillation from a teacher's largest logits.  The contractions, their tiles and their launches are those of the plain
// cross-entropy; what differs is what is taken from a tile of logits and what the logits' gradient is.
//
// Notation of a row: z logits, y = c tanh(z / c) (y = z without a cap), T the temperature, "entries" the vocabulary entries that
// the teacher gives, "others" the rest.
//
//   forward   k_entries        the teacher's entries of every row in ascending order, and where each vocabulary tile's begin (for
//                              tiles of more than 32 rows; others find them as they need them: TileEntries)
//             (logits)         ObjEpilogue: the label's y and the entries' z out of the accumulators; partial log-sum-exps of the
//                              others alone, at 1 / T and, where a row needs both, at 1
//             k_obj_finalize   log-sum-exps, losses, what the backward needs of each row and at each entry
//             k_obj_loss       the loss, in a fixed order (small calls: with the rows' losses, by k_obj_finalize or k_obj_finalize_one)
//   backward  (logits again)   ObjGrad: every entry of a row as two coefficients times exponentials
//             k_obj_entries    the teacher's entries put into the block of dlogits
//
// The others' log-sum-exp is formed without the entries, not as a difference: where the student gives nearly everything to the
// entries a difference of float32 numbers would leave nothing of the share of the others.
#pragma once
#include <type_traits>

#include "mst_small_kernels.hpp"

namespace mst {

constexpr int kMaxEntries = 256;            // of a row of the teacher
constexpr int kNoEntry = 0x7fffffff;        // sorts behind every entry

// What the backward call needs, at the front of the caller's `saved`.
struct ObjHeader {
  long long n_valid;                        // rows that count; -1: an index out of range
  long long n_divisor;                      // what the gradient's sums are divided by, a double's bits (-1 again, 0 where no row counts)
  float cap, exponent, exponent_label;      // log2(e) / T of the (first) exponential, log2(e) of the second
  int two;                                  // rows have two exponentials
};

// Of one row, for the backward: the gradient of y_v is
//   at * exp((y_v - base) / T) + row2.at * exp(y_v - row2.base) - [v == label] label_term
// at every entry that is not the teacher's; the second exponential only where there are two (ObjRow2).
struct ObjRow { float base, at, label_term; int label; };
struct ObjRow2 { float base, at; };

// y = c tanh(z / c) and its slope 1 - tanh^2, x = z / c, without cancellation anywhere:
//   |x| < 1/2   tanh x = x + x p, p = x^2 q(x^2), with q of degree 3 the polynomial whose largest relative error in tanh is least (1.5e-8, by
//               weighted least squares until the errors' peaks are equal); 1 - tanh^2 as it stands, tanh^2 being at most 0.22.  1.3 half steps of y.
//   elsewhere   by u = 1 / (1 + exp(2 |x|)) <= 0.27: tanh |x| = 1 - 2 u, slope 4 u (1 - u).  5 half steps of y.
// Formed as 1 - 2 u throughout, y is half a step of the cap off whatever z is: 0.12 at a cap of 1e6.  The polynomial alone costs less than
// exp2 and the reciprocal, both ways and a choice more; 8192 x 3584 x 128000, logits of 2.5, us, forward and backward: no cap 4950, 16300; as
// 1 - 2 u 5125, 16600 at any cap; so 5080, 16600 at caps of 50 and 30, 5320, 17200 at 10 and 2.
struct Cap {
  float c, by_c, scale;                // 2 log2(e) / c
  __device__ __forceinline__ explicit Cap(float cap) : c(cap), by_c(1.f / cap), scale(2.f * kLog2e / cap) {}
  __device__ __forceinline__ bool near(float z) const { return __builtin_fabsf(z) < 0.5f * c; }
  __device__ __forceinline__ float p(float x) const {
    const float w = x * x;
    float q = 1.724154502e-2f;
    q = __builtin_fmaf(q, w, -5.304551497e-2f);
    q = __builtin_fmaf(q, w, 1.332587898e-1f);
    q = __builtin_fmaf(q, w, -3.333314359e-1f);
    return w * q;
  }
  __device__ __forceinline__ float u(float z) const { return __builtin_amdgcn_rcpf(1.f + fast_exp2(__builtin_fabsf(z) * scale)); }
  // kNear: |z| < c / 2 is known; else both ways, the same bits
  template <bool kNear> __device__ __forceinline__ float y(float z) const {
    const float at_0 = __builtin_fmaf(z, p(z * by_c), z);
    if (kNear) return at_0;
    const float far = __builtin_copysignf(c - 2.f * c * u(z), z);
    return near(z) ? at_0 : far;
  }
  template <bool kNear> __device__ __forceinline__ float slope(float z) const {
    const float x = z * by_c, t = __builtin_fmaf(x, p(x), x), at_0 = __builtin_fmaf(-t, t, 1.f);
    if (kNear) return at_0;
    const float v = u(z);
    return near(z) ? at_0 : 4.f * v * (1.f - v);
  }
};

// merge_lse for sums of exp2(exponent (y - m)), and a second sum beside the first at another exponent
__device__ __forceinline__ void merge_sums(float& m, float& l, float& k, float m2, float l2, float k2, float exponent, float exponent_label,
                                           bool two) {
  const float mm = fmaxf(m, m2), a = m - mm, b = m2 - mm;
  l = __builtin_fmaf(l, fast_exp2(a * exponent), l2 * fast_exp2(b * exponent));
  if (two) k = __builtin_fmaf(k, fast_exp2(a * exponent_label), k2 * fast_exp2(b * exponent_label));
  m = mm;
}

// ---------------------------------------------------------------------------
// forward epilogue
// ---------------------------------------------------------------------------
struct ObjTile {
  const int* labels_c;                 // null: none
  float2* part;                        // [n_vt][part_stride] (maximum, sum) of the others
  float* part_label;                   // the sum at the second exponent; null: rows have one
  size_t part_stride;
  float* tgt;                          // y of the label, unless it is an entry
  int K;                               // 0: no teacher
  int* index;                          // [rows][K] the entries, kNoEntry where there is none
  float* entry_z;                      // [rows][K] their logits
  const unsigned short* starts;        // [n_vt + 1][part_stride]: entries before a tile, with `index` ascending; null where the tile
                                       // finds its entries among the caller's and writes `index` and `info` (TileEntries)
  const int* index_in_c;
  int* info;
  float cap, exponent, exponent_label;
};

// f(row, place in its list, index) for all entries of a tile's rows, [rows][K] from `index` on.  A thread's first ones can be loaded
// long before (first_entries).
constexpr int kEntriesAtOnce = 8;
struct FirstEntries { int v[kEntriesAtOnce]; };
template <int kThreadsOfTile>
__device__ __forceinline__ FirstEntries load_entries(const int* __restrict__ index, int n, int i0) {
  FirstEntries e;
#pragma unroll
  for (int b = 0; b < kEntriesAtOnce; ++b) e.v[b] = index[i0 + b * kThreadsOfTile < n ? i0 + b * kThreadsOfTile : n - 1];
  return e;
}
template <int kThreadsOfTile, class F>
__device__ __forceinline__ void each_entry(const FirstEntries& first, const int* __restrict__ index, int rows, int K, F f) {
  const int n = rows * K;
  const float by_k = 1.f / (float)K;
  FirstEntries e = first;
  for (int i0 = threadIdx.x; i0 < n;) {
#pragma unroll
    for (int b = 0; b < kEntriesAtOnce; ++b) {
      const int i = i0 + b * kThreadsOfTile;
      const int r = (int)(((float)i + 0.5f) * by_k);       // i / K: i < 2^15, K <= 2^8, half of 1 / K is more than the product is off by
      if (i < n) f(r, i - r * K, e.v[b]);
    }
    i0 += kEntriesAtOnce * kThreadsOfTile;
    if (i0 < n) e = load_entries<kThreadsOfTile>(index, n, i0);
  }
}

// A tile's entries without a launch before it, for tiles of up to 32 rows, which are all in one round of workgroups: its threads look
// through the entries of its rows and note in LDS which of the tile's kWidth vocabulary entries are the teacher's (a bit each) and at
// which place of the row's list (the first, where an index comes twice).  The tile that has an entry writes what the following kernel
// reads of it, the first tile also what is no entry.  512 x 256 x 4096 with 20 entries: 8.6 us of a launch of sorting, 3 us here.
template <int kRows, int kWidth, int kThreadsOfTile>
struct TileEntries {
  static constexpr int kWords = kWidth / 32;
  static constexpr int kBytes = kRows * (kWords + 2 * kWidth) * 4;
  static_assert(kRows * kMaxEntries <= 1 << 15 && kBytes % 16 == 0, "each_entry");
  unsigned* bits;                      // [kRows][kWords]
  int* place;                          // [kRows][kWidth], where there is a bit
  float* z;                            // [kRows][kWidth]: for the tile's logits where there is a bit
  // smem: kBytes, 16-byte aligned, that nobody uses; all threads of the workgroup
  __device__ __forceinline__ TileEntries(char* smem, const ObjTile& e, const FirstEntries& first, int s0, int rows, int v0, int V, bool first_tile)
      : bits(reinterpret_cast<unsigned*>(smem)), place(reinterpret_cast<int*>(bits + kRows * kWords)),
        z(reinterpret_cast<float*>(place + kRows * kWidth)) {
    for (int i = threadIdx.x; i < kRows * kWords; i += kThreadsOfTile) bits[i] = 0;
    for (int i = threadIdx.x; i < kRows * kWidth / 4; i += kThreadsOfTile)
      reinterpret_cast<int4*>(place)[i] = make_int4(kNoEntry, kNoEntry, kNoEntry, kNoEntry);
    const int here = rows - s0 < kRows ? rows - s0 : kRows;
    if (first_tile)
      for (int r = threadIdx.x; r < here; r += kThreadsOfTile) e.info[s0 + r] = e.K;
    __syncthreads();
    each_entry<kThreadsOfTile>(first, e.index_in_c + (size_t)s0 * e.K, here, e.K, [&](int r, int k, int v) {
      if ((unsigned)(v - v0) >= (unsigned)kWidth || v >= V) return;
      atomicMin(place + r * kWidth + v - v0, k);
      atomicOr(bits + r * kWords + (v - v0) / 32, 1u << ((v - v0) & 31));
    });
    __syncthreads();
  }
  // behind the tile's logits in LDS
  __device__ __forceinline__ void write(const ObjTile& e, const FirstEntries& first, int s0, int rows, int v0, int V, bool first_tile) const {
    __syncthreads();
    const int here = rows - s0 < kRows ? rows - s0 : kRows;
    const size_t from = (size_t)s0 * e.K;
    each_entry<kThreadsOfTile>(first, e.index_in_c + from, here, e.K, [&](int r, int k, int v) {
      const size_t at = from + (size_t)r * e.K + k;
      if ((unsigned)(v - v0) < (unsigned)kWidth && v < V) {
        const int in = r * kWidth + v - v0;
        const bool kept = place[in] == k;
        e.index[at] = kept ? v : kNoEntry;
        if (kept) e.entry_z[at] = z[in];
      } else if (first_tile && (unsigned)v >= (unsigned)V) {
        e.index[at] = kNoEntry;
        if (v >= V) e.info[s0 + r] = -1;             // behind e.K, with barriers in between
      }
    });
  }
};

// kWhat: what is known when compiled, 0 or kObjCap for calls without a teacher; kObjAny asks the arguments.
// Known against asked, us: 16384 x 3584 x 256000 with a cap 20780, 20980; with a teacher the same.
constexpr int kObjCap = 1, kObjAny = 2;
template <int kWhat>
struct ObjEpilogue : ObjTile {
  typedef ObjEpilogue<kObjAny> Small;          // of the smaller tiles
  static constexpr bool kWhole = false;
  ObjEpilogue() = default;
  explicit ObjEpilogue(const ObjTile& t) : ObjTile(t) {}

  // what is on its way during a small tile's main loop
  template <class C> static constexpr bool has_early() { return C::EB <= 32; }
  typedef FirstEntries Early;
  template <class C>
  __device__ __forceinline__ Early early(int rows, int s0) const {
    if constexpr (has_early<C>())
      if (K) return load_entries<C::kThreads>(index_in_c + (size_t)s0 * K, (rows - s0 < C::EB ? rows - s0 : C::EB) * K, threadIdx.x);
    return Early();
  }

  template <class C>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[C::TA][C::TB], int rows, int V, int vt, int s0, int wa, int wb, int lane, char* smem,
                                             const Early& first_entries = Early()) const {
    constexpr int TA = C::TA, TB = C::TB, kPer = 4 * TA, kWaveV = 16 * TA;    // vocabulary entries of a lane, of a wave
    constexpr bool kSorted = !has_early<C>();          // entries from k_entries
    typedef TileEntries<C::EB, C::EA, C::kThreads> Found;
    const bool teacher = kWhat == kObjAny && K > 0, two = kWhat == kObjAny && part_label != nullptr;
    const int v0 = vt * C::EA;
    const int g = lane >> 4, c = lane & 15;
    const int va = v0 + wa * kWaveV + kPer * g;        // a lane's consecutive entries of each of its TB rows
    int y_u[TB], from[TB], to[TB];                     // on their way meanwhile
#pragma unroll
    for (int u = 0; u < TB; ++u) {
      const int s_local = s0 + wb * (16 * TB) + 16 * u + c, s_in = s_local < rows ? s_local : rows - 1;
      y_u[u] = labels_c ? labels_c[s_in] : -1;
      from[u] = teacher && kSorted ? starts[(size_t)vt * part_stride + s_in] : 0;
      to[u] = teacher && kSorted ? starts[(size_t)(vt + 1) * part_stride + s_in] : 0;
    }
    float* xch = reinterpret_cast<float*>(smem);       // [wb][u][16] triples of the wa == 1 waves; the main loop ended with a barrier
    const bool bends = kWhat == kObjAny ? cap > 0.f : kWhat == kObjCap;
    // Bit t / kSame: some of the wave's logits acc[t] and of the next kSame - 1, 16 of a lane, are far from 0 (seldom), before any is masked.
    constexpr int kSame = TB >= 4 ? 1 : TA * TB >= 4 ? 4 / TB : TA;
    static_assert(TA % kSame == 0, "whole groups");
    unsigned far = 0;
    if (bends) {
      const Cap bend(cap);
#pragma unroll
      for (int t0 = 0; t0 < TA; t0 += kSame) {
        float top = 0.f;
#pragma unroll
        for (int t = t0; t < t0 + kSame; ++t)
#pragma unroll
          for (int u = 0; u < TB; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, __builtin_fabsf(acc[t][u][r]));
        if (__any(!bend.near(top))) far |= 1u << (t0 / kSame);
      }
    }
    // The entries' logits out of the accumulators, in which they are masked then.  mine: bit i, entry va + i is the teacher's.
    auto take = [&](int u, unsigned mine, auto put) {
      if (!__any(mine != 0)) return;
#pragma unroll
      for (int t = 0; t < TA; ++t) {
        if (!__any((mine >> (4 * t)) & 15u)) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if ((mine >> (4 * t + r)) & 1u) {
            put(4 * t + r, acc[t][u][r]);
            acc[t][u][r] = kMasked;
          }
      }
    };
    if (teacher) {
      if constexpr (kSorted) {
        // The first entries of all rows at once: one after the other each would wait for the one before.
        constexpr int kAtOnce = 4;
        int entry[TB][kAtOnce];
#pragma unroll
        for (int u = 0; u < TB; ++u) {
          const int s_local = s0 + wb * (16 * TB) + 16 * u + c;
          if (s_local >= rows) to[u] = 0;
          const int* const row = index + (size_t)(s_local < rows ? s_local : rows - 1) * K;
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) entry[u][i] = row[from[u] + i < K ? from[u] + i : K - 1];
        }
#pragma unroll
        for (int u = 0; u < TB; ++u) {
          const int s_local = s0 + wb * (16 * TB) + 16 * u + c;
          unsigned mine = 0;
          int first = 0;                               // place of the lowest of them
          auto note = [&](int e, int v) {
            const int rel = v - va;
            if ((unsigned)rel < (unsigned)kPer && e < to[u]) {
              if (!mine) first = e;
              mine |= 1u << rel;
            }
          };
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) note(from[u] + i, entry[u][i]);
          for (int e0 = from[u] + kAtOnce; e0 < to[u]; e0 += kAtOnce) {
            int more[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) more[i] = index[(size_t)s_local * K + (e0 + i < K ? e0 + i : K - 1)];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) note(e0 + i, more[i]);
          }
          float* out = entry_z + (size_t)(s_local < rows ? s_local : rows - 1) * K + first;      // a lane's entries follow each other
          take(u, mine, [&](int, float z) { *out++ = z; });
        }
      } else {
        static_assert(Found::kBytes + 2 * C::EB * 12 <= C::kLds, "beside the triples");
        const Found found(smem, *this, first_entries, s0, rows, v0, V, vt == 0);
        xch = reinterpret_cast<float*>(smem + Found::kBytes);
#pragma unroll
        for (int u = 0; u < TB; ++u) {
          const int r = wb * (16 * TB) + 16 * u + c;   // past the last row: no bits
          float* const out = found.z + r * C::EA + va - v0;
          const unsigned word = found.bits[r * Found::kWords + (va - v0) / 32];
          take(u, (word >> ((va - v0) & 31)) & (0xffffffffu >> (32 - kPer)), [&](int i, float z) { out[i] = z; });
        }
        found.write(*this, first_entries, s0, rows, v0, V, vt == 0);
      }
    }
    if (bends) {                       // behind the entries, whose slopes need the logits themselves
      const Cap bend(cap);
#pragma unroll
      for (int t0 = 0; t0 < TA; t0 += kSame) {
        auto all = [&](auto near) {
          constexpr bool kNear = decltype(near)::value;          // then the polynomial makes -infinity of kMasked, as good a mask
#pragma unroll
          for (int t = t0; t < t0 + kSame; ++t)
#pragma unroll
            for (int u = 0; u < TB; ++u)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float z = acc[t][u][r], y = bend.template y<kNear>(z);
                acc[t][u][r] = !kNear && teacher && z == kMasked ? kMasked : y;
              }
        };
        if ((far >> (t0 / kSame)) & 1u) all(std::false_type()); else all(std::true_type());
      }
    }
    if (v0 + C::EA > V) {
#pragma unroll
      for (int t = 0; t < TA; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (va + 4 * t + r >= V) {
#pragma unroll
            for (int u = 0; u < TB; ++u) acc[t][u][r] = kMasked;
          }
    }
    float m_u[TB], l_u[TB], k_u[TB];
#pragma unroll
    for (int u = 0; u < TB; ++u) {
      float m = kMasked, l = 0.f, k = 0.f;
#pragma unroll
      for (int t = 0; t < TA; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[t][u][r]);
#pragma unroll
      for (int t = 0; t < TA; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) l += fast_exp2((acc[t][u][r] - m) * exponent);
      if (two) {           // at T = 2 and 4 a power of the first, to no gain: 8192 x 4096 x 128256 5850 us with exponentials, 5888 with squares
#pragma unroll
        for (int t = 0; t < TA; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) k += fast_exp2((acc[t][u][r] - m) * exponent_label);
      }
#pragma unroll
      for (int o = 16; o <= 32; o <<= 1)
        merge_sums(m, l, k, __shfl_xor(m, o), __shfl_xor(l, o), two ? __shfl_xor(k, o) : 0.f, exponent, exponent_label, two);
      m_u[u] = m; l_u[u] = l; k_u[u] = k;

      // y of the label straight from the accumulator that holds it
      const int s_local = s0 + wb * (16 * TB) + 16 * u + c;
      const int y = s_local < rows ? y_u[u] : -1;
      const int rel = y - va;
      if ((unsigned)rel < (unsigned)kPer && y < V) {
        const int t_sel = rel >> 2, r_sel = rel & 3;
        float val = 0.f;
#pragma unroll
        for (int t = 0; t < TA; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (t == t_sel && r == r_sel) val = acc[t][u][r];
        tgt[s_local] = val;
      }
    }
    if (wa == 1 && lane < 16) {
#pragma unroll
      for (int u = 0; u < TB; ++u) {
        float* at = xch + ((wb * TB + u) * 16 + lane) * 3;
        at[0] = m_u[u]; at[1] = l_u[u]; at[2] = k_u[u];
      }
    }
    __syncthreads();
    if (wa == 0 && lane < 16) {
#pragma unroll
      for (int u = 0; u < TB; ++u) {
        const float* at = xch + ((wb * TB + u) * 16 + lane) * 3;
        merge_sums(m_u[u], l_u[u], k_u[u], at[0], at[1], at[2], exponent, exponent_label, two);
        const int s_local = s0 + wb * (16 * TB) + 16 * u + lane;
        if (s_local >= rows) continue;
        part[(size_t)vt * part_stride + s_local] = make_float2(m_u[u], l_u[u]);
        if (two) part_label[(size_t)vt * part_stride + s_local] = k_u[u];
      }
    }
  }
};

// Calls that have tiles of 32 rows and 256 vocabulary entries for half of the compute units or fewer: with up to 32 rows W is read once,
// which is all that takes time, and a compute unit alone does not get its share of the memory's bandwidth; with more a few workgroups take
// the K loop's steps one by one.  Tiles of 64, two workgroups on a compute unit where there are as many.  Whole calls, us, tiles of 256
// and these: 33 rows, V = 300: d = 512 9.8, 7.8; 4096 29.1, 17.2; 500 rows, V = 1000: 1536 16.3, 12.0; with 30 entries 23.9, 18.7; but where
// tiles of 256 are for all compute units, 512 rows, V = 4096, d = 1024 15.1, 22.2.  Forward of 16 rows, us, with tiles of 256, of 128 (lone
// ones, eight stages) and these: d = 4096, V = 32768 68.2, 64.6, 58.1 (4.6 TB/s); 16000 54.3, 38.0, 33.0; 8000 30.7, 22.1, 19.2; d = 2048,
// V = 4000 19.6, 15.8, 13.4.
// (With both operands from memory straight into registers, a wave to 16 vocabulary entries: 57.8 for one row, 71.4 for 16.)
typedef CfgSmall<2, 1, 6, 6, true> TileFew;

// ---------------------------------------------------------------------------
// The teacher's entries of a group of rows in ascending order.  A wave sorts a row, P entries a lane, with a bitonic network on
// (index, place) in 64 bits: of entries with the same index the first comes first and the others are dropped.  An index below 0 is
// no entry; one at or behind V makes the row bad.
//   index, logit [rows][K] (float32), the rest of a row kNoEntry; info[row] = entries, or -1 where the row is bad
//   starts [n_vt + 1][stride]: entries before vocabulary entry 256 vt
// 32768 rows of 256: 510 us with every entry compared to all others of its row, in LDS.
// ---------------------------------------------------------------------------
constexpr int kEntryRows = 16;              // of a workgroup, one wave each: 32-byte pieces of starts
template <int P>
__device__ __forceinline__ void sort_entries(unsigned long long (&x)[P], int lane) {
  auto order = [](unsigned long long& a, unsigned long long& b, bool up) {
    const bool swap = (b < a) == up;
    const unsigned long long t = a;
    a = swap ? b : a;
    b = swap ? t : b;
  };
#pragma unroll
  for (int k = 2; k <= 64 * P; k *= 2)
#pragma unroll
    for (int j = k / 2; j > 0; j /= 2) {
      if (j >= P) {
        const bool lower = (lane & (j / P)) == 0;
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const unsigned long long other = __shfl_xor(x[i], j / P);
          const bool up = ((lane * P + i) & k) == 0;
          x[i] = (other < x[i]) == (up == lower) ? other : x[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (!(i & j)) order(x[i], x[i | j], ((lane * P + i) & k) == 0);
      }
    }
}
template <int P>
__global__ __launch_bounds__(64 * kEntryRows) void k_entries(
    const int* __restrict__ index_in, const void* __restrict__ logit_in, int logit_bf16, int rows, int K, int V, int n_vt,
    int* __restrict__ index, float* __restrict__ logit, int* __restrict__ info, unsigned short* __restrict__ starts, size_t stride) {
  __shared__ int key_sh[kEntryRows][64 * P];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int s = blockIdx.x * kEntryRows + w, s_in = s < rows ? s : rows - 1;
  unsigned long long x[P];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = lane * P + i;
    int v = e < K ? index_in[(size_t)s_in * K + e] : -1;
    bad |= v >= V;
    if ((unsigned)v >= (unsigned)V) v = kNoEntry;
    x[i] = ((unsigned long long)(unsigned)v << 8) | (unsigned)e;
  }
  bad = __any(bad);
  sort_entries<P>(x, lane);
  int v[P];
  bool keep[P];
  int before = 0, n = 0;                      // entries that are kept: in lanes below, in all
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = (int)(x[i] >> 8);
  const int last_below = __shfl_up(v[P - 1], 1);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const bool again = i ? v[i] == v[i ? i - 1 : 0] : lane > 0 && v[0] == last_below;
    keep[i] = v[i] != kNoEntry && !again;
    const unsigned long long all = __ballot(keep[i]);
    before += __builtin_popcountll(all & ((1ull << lane) - 1));
    n += __builtin_popcountll(all);
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int place = keep[i] ? before : n + lane * P + i - before;      // what is dropped goes behind the rest
    before += keep[i];
    key_sh[w][place] = keep[i] ? v[i] : kNoEntry;
    if (place >= K || s >= rows) continue;
    const size_t to = (size_t)s * K + place, at = (size_t)s * K + (int)(x[i] & 255);
    index[to] = keep[i] ? v[i] : kNoEntry;
    if (keep[i]) logit[to] = logit_bf16 ? (float)static_cast<const __bf16*>(logit_in)[at] : static_cast<const float*>(logit_in)[at];
  }
  if (lane == 0 && s < rows) info[s] = bad ? -1 : n;
  __syncthreads();
  // by bisection
  const int r = threadIdx.x % kEntryRows, row = blockIdx.x * kEntryRows + r;
  if (row >= rows) return;
  for (int vt = threadIdx.x / kEntryRows; vt <= n_vt; vt += 64) {
    const int v0 = vt < n_vt ? vt * kTile : kNoEntry;
    int lo = 0, hi = K;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (key_sh[r][mid] < v0) lo = mid + 1; else hi = mid;
    }
    starts[(size_t)vt * stride + row] = (unsigned short)lo;
  }
}

// ---------------------------------------------------------------------------
// Per row: log-sum-exps, losses, and what the backward needs.  A workgroup owns 16 rows; first its 16 groups of threads each
// fold every 16th vocabulary tile of each row (as k_lse_finalize), then 16 neighbouring lanes have a row each.  All sums in a
// fixed order.
// ---------------------------------------------------------------------------
struct ObjFinal {
  const float2* part;
  const float* part_label;
  size_t part_stride;
  int n_vt, rows, V, K;
  const float* tgt;
  const int* labels_c;
  const float* weights_c;
  int ignore_index;
  const int* index;                   // [rows][K] (kNoEntry: none), and the entries' logits, the teacher's and the student's
  const float* logit;                 // null: the caller's, in the order of its list
  const void* logit_in_c;
  int logit_bf16;
  const float* entry_z;
  const int* info;
  const float* teacher_lse_c;
  float cap, exponent, exponent_label, inv_t;
  double inv_t_64;
  float label_coef, teacher_coef, z_coef, temperature;
  float label_slope, teacher_slope, z_slope;      // of the gradient, in units of ObjLoss::unit
  float *nll_c, *kd_c, *lse_c;        // outputs, each may be null
  float2* row_loss_c;                 // the row's loss, and as an integer's bits 1: it counts, -1: an index out of range
  ObjRow* rows_c;                     // null: no backward follows
  ObjRow2* rows2_c;
  int* saved_index_c;
  float* saved_at_c;
};
// Logarithm with 64-bit steps: x = m 2^e, m in [1/sqrt 2, sqrt 2), log m = 2 artanh((m - 1) / (m + 1)) by its series, whose first term left
// out is below 2e-12 of it.  The finalize kernel of 512 rows of 20 entries takes 6.7 us with it and 8.3 us with the library's 64-bit log.
__device__ __forceinline__ double log_64(float x) {
  if (!(x >= 1.17549435e-38f && x < __builtin_inff())) return (double)logf(x);
  const int bits = __builtin_bit_cast(int, x), e = (bits - 0x3f3504f3) >> 23;            // 0x3f3504f3: 1 / sqrt 2
  const double m = (double)__builtin_bit_cast(float, bits - (e << 23));
  double r = (double)__builtin_amdgcn_rcpf((float)(m + 1.0));
  r *= __builtin_fma(-(m + 1.0), r, 2.0);
  const double a = (m - 1.0) * r, z = a * a;
  double f = 1.0 / 13.0;
  f = __builtin_fma(f, z, 1.0 / 11.0);
  f = __builtin_fma(f, z, 1.0 / 9.0);
  f = __builtin_fma(f, z, 1.0 / 7.0);
  f = __builtin_fma(f, z, 1.0 / 5.0);
  f = __builtin_fma(f, z, 1.0 / 3.0);
  f = __builtin_fma(f, z, 1.0);
  return __builtin_fma(2.0 * a, f, (double)e * 0.69314718055994530942);
}
// exp of a logarithm in 64 bits: that of its float32 part, and what that leaves as a factor
__device__ __forceinline__ float exp_of(double x) {
  if (!(__builtin_fabs(x) <= 1000.0)) return x < 0.0 ? 0.f : expf((float)x);      // NaN and infinities, and what float32 has no number for
  const float hi = (float)x, lo = (float)(x - (double)hi);
  return __builtin_fmaf(expf(hi), lo, expf(hi));
}
// q (exp(w) - 1 - w) with q exp(w) = p: around 0 by the series of the bracket, whose first term left out is 1 / 40320 w^8; q (exp(w) - 1)
// likewise.  Elsewhere by p, as exp(w) has no float32 where q is next to nothing.
__device__ __forceinline__ float above_tangent(float q, float p, float w) {
  if (q == 0.f) return p;
  if (__builtin_fabsf(w) < 0.25f) {
    float s = 1.f / 5040.f;
    s = __builtin_fmaf(s, w, 1.f / 720.f);
    s = __builtin_fmaf(s, w, 1.f / 120.f);
    s = __builtin_fmaf(s, w, 1.f / 24.f);
    s = __builtin_fmaf(s, w, 1.f / 6.f);
    s = __builtin_fmaf(s, w, 0.5f);
    return q * (s * w * w);
  }
  return (float)((double)p - (double)q - (double)q * (double)w);
}
__device__ __forceinline__ float share_less(float q, float p, float w) { return __builtin_fabsf(w) < 1.f ? q * expm1f(w) : p - q; }

// What the loss needs besides the rows'.
struct ObjLoss {
  long long divisor;
  double unit;                        // the gradient's: its rows, in bf16, are in units of it
  ObjHeader head;
  ObjHeader* saved;                   // null: no backward follows
  float* loss;
  long long* n_valid;
};
__device__ __forceinline__ void write_loss(const ObjLoss& o, double sum, long long n, int bad) {
  const long long divisor = bad ? -1 : n == 0 ? 0 : o.divisor > 0 ? o.divisor : n;
  *o.loss = bad ? __builtin_nanf("") : n == 0 ? 0.f : (float)(sum / (double)divisor);
  if (o.n_valid) *o.n_valid = bad ? -1 : n;
  if (!o.saved) return;
  o.saved->n_valid = bad ? -1 : n;
  o.saved->n_divisor = divisor > 0 ? __builtin_bit_cast(long long, (double)divisor / o.unit) : divisor;
  o.saved->cap = o.head.cap;
  o.saved->exponent = o.head.exponent;
  o.saved->exponent_label = o.head.exponent_label;
  o.saved->two = o.head.two;
}
constexpr int kObjRows = 16, kObjGroups = 16;

// Over the 16 lanes of a row, by rotations within them: every lane adds the same pairs, so all have the same bits.
template <int kBy> __device__ __forceinline__ int rotate16(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + kBy, 0xf, 0xf, true); }
template <int kBy> __device__ __forceinline__ float rotate16(float x) {
  return __builtin_bit_cast(float, rotate16<kBy>(__builtin_bit_cast(int, x)));
}
template <int kBy> __device__ __forceinline__ double rotate16(double x) {
  int2 h = __builtin_bit_cast(int2, x);
  h.x = rotate16<kBy>(h.x);
  h.y = rotate16<kBy>(h.y);
  return __builtin_bit_cast(double, h);
}
__device__ __forceinline__ float max16(float x) {
  x = fmaxf(x, rotate16<8>(x));
  x = fmaxf(x, rotate16<4>(x));
  x = fmaxf(x, rotate16<2>(x));
  return fmaxf(x, rotate16<1>(x));
}
template <class X> __device__ __forceinline__ X sum16(X x) {
  x += rotate16<8>(x);
  x += rotate16<4>(x);
  x += rotate16<2>(x);
  return x + rotate16<1>(x);
}

// kAll: the rows are all of the call's, whose loss is formed here too (one launch less).  P: entries of a lane, all of which are
// on their way with the first loads (read in a loop for each use, 512 rows of 20 entries took 8.6 us).
template <bool kAll, int P>
__global__ __launch_bounds__(kObjRows * kObjGroups) void k_obj_finalize(ObjFinal a, ObjLoss o) {
  __shared__ float sh[kObjRows][kObjGroups][3];
  const bool two = a.part_label != nullptr;
  const int r = threadIdx.x >> 4, lane = threadIdx.x & 15;
  const int s = blockIdx.x * kObjRows + r;
  const bool in = s < a.rows;
  const int s_in = in ? s : a.rows - 1;
  const size_t at0 = (size_t)s_in * a.K;
  int v_p[P ? P : 1];
  float z_p[P ? P : 1], t_p[P ? P : 1];                          // of the row's entries lane, lane + 16, ...
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = lane + 16 * i, e_in = e < a.K ? e : a.K - 1;
    const int v = a.index[at0 + e_in];
    z_p[i] = a.entry_z[at0 + e_in];
    t_p[i] = a.logit ? a.logit[at0 + e_in] : a.logit_bf16 ? (float)static_cast<const __bf16*>(a.logit_in_c)[at0 + e_in]
                                                          : static_cast<const float*>(a.logit_in_c)[at0 + e_in];
    v_p[i] = e < a.K ? v : kNoEntry;
  }
  const int y = a.labels_c ? a.labels_c[s_in] : a.ignore_index;
  const float weight = a.weights_c ? a.weights_c[s_in] : 1.f;
  const bool bad_entry = P && a.info[s_in] < 0;
  const bool given = P && a.teacher_lse_c != nullptr;
  const float given_lse = given ? a.teacher_lse_c[s_in] : 0.f;
  const float tgt = a.tgt[s_in];
  {
    const int r = threadIdx.x & (kObjRows - 1), g = threadIdx.x / kObjRows;
    const int s = blockIdx.x * kObjRows + r;
    float m = kMasked, l = 0.f, k = 0.f;
    if (s < a.rows) {
      constexpr int kBatch = 16;
      for (int v0 = g; v0 < a.n_vt; v0 += kBatch * kObjGroups) {
        float2 p[kBatch];
        float q[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int vt = v0 + i * kObjGroups;
          p[i] = vt < a.n_vt ? a.part[(size_t)vt * a.part_stride + s] : make_float2(kMasked, 0.f);
          q[i] = two && vt < a.n_vt ? a.part_label[(size_t)vt * a.part_stride + s] : 0.f;
        }
        float mm = m;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) mm = fmaxf(mm, p[i].x);
        l *= fast_exp2((m - mm) * a.exponent);
        k *= fast_exp2((m - mm) * a.exponent_label);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) l = __builtin_fmaf(p[i].y, fast_exp2((p[i].x - mm) * a.exponent), l);
        if (two) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) k = __builtin_fmaf(q[i], fast_exp2((p[i].x - mm) * a.exponent_label), k);
        }
        m = mm;
      }
    }
    sh[r][g][0] = m; sh[r][g][1] = l; sh[r][g][2] = k;
  }
  __syncthreads();
  // the others
  const float m_lane = sh[r][lane][0];
  const float m = max16(m_lane);
  const float l = sum16(sh[r][lane][1] * fast_exp2((m_lane - m) * a.exponent));
  const float k = two ? sum16(sh[r][lane][2] * fast_exp2((m_lane - m) * a.exponent_label)) : 0.f;
  const bool others = m > 0.5f * kMasked;                        // there are some

  // the entries
  auto entries = [&](auto f) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (v_p[i] != kNoEntry) f(i);
  };
  float y_p[P ? P : 1];
#pragma unroll
  for (int i = 0; i < P; ++i) y_p[i] = a.cap > 0.f ? Cap(a.cap).y<false>(z_p[i]) : z_p[i];
  float my = kMasked, mt = kMasked;
  int some = 0;
  entries([&](int i) {
    my = fmaxf(my, y_p[i]);
    mt = fmaxf(mt, t_p[i]);
    some = 1;
  });
  my = max16(my);
  mt = max16(mt);
  some = sum16(some);
  float ly = 0.f, ky = 0.f, lt = 0.f;
  entries([&](int i) {
    const float y = y_p[i] - my;
    ly += fast_exp2(y * a.exponent);
    if (two) ky += fast_exp2(y * a.exponent_label);
    lt += expf((t_p[i] - mt) * a.inv_t);
  });
  ly = sum16(ly);
  ky = sum16(ky);
  lt = sum16(lt);
  const bool labelled = a.labels_c && y != a.ignore_index;
  const bool valid = labelled && (unsigned)y < (unsigned)a.V;
  float y_entry = 0.f;                                           // the label's logit where it is an entry
  int is_entry = 0;
  if (valid)
    entries([&](int i) {
      if (v_p[i] == y) y_entry = y_p[i], is_entry = 1;
    });
  y_entry = sum16(y_entry);
  is_entry = sum16(is_entry);

  // log-sum-exps, as maximum and logarithm of the sum: at 1 / T (m_all / T + log_all), and at 1 (m_all + log_label)
  const float m_all = fmaxf(m, my);
  const float l_all = l * fast_exp2((m - m_all) * a.exponent) + ly * fast_exp2((my - m_all) * a.exponent);
  const float k_all = two ? k * fast_exp2((m - m_all) * a.exponent_label) + ky * fast_exp2((my - m_all) * a.exponent_label) : l_all;
  const double log_all = log_64(l_all);
  const float log_label = two ? logf(k_all) : (float)log_all;
  const float lse = m_all + log_label;
  const float base = m + a.temperature * logf(l);                // T times the others' log-sum-exp at 1 / T
  const double log_share = ((double)m - (double)m_all) * a.inv_t_64 + (log_64(l) - log_all);       // of the others' share

  const float nll = valid ? (m_all - (is_entry ? y_entry : tgt)) + log_label : 0.f;

  // the teacher's shares; `rest`: what it leaves to the others
  const bool taught = some > 0 && (given || !(mt <= 0.5f * kMasked) || lt != lt);      // a maximum passes over NaN, a sum does not
  // The divergence is formed of parts that are 0 where a share is the teacher's and else positive: with w = log p - log q
  //   sum q (log q - log p) = sum q (exp(w) - 1 - w) + (sum q - sum p),
  // and the shares of both add up to 1.  What a log-sum-exp is off by changes a part by (p - q) times that and not by q times; softened
  // distributions (T = 4, 9 of 14144 entries) leave a divergence of 0.002 of logarithms of 10, and float32 differences of these left 2e-4
  // of it.  The logarithms of shares are differences in 64 bits for the same reason.
  const double log_lt = given ? 0.0 : log_64(lt);
  float q_p[P ? P : 1], p_p[P ? P : 1], w_p[P ? P : 1];         // shares, the teacher's and the student's, and w
  double sum_q = 0.0, kd_64 = 0.0;
  entries([&](int i) {
    const double log_q = given ? (double)t_p[i] * a.inv_t_64 - (double)given_lse : ((double)t_p[i] - (double)mt) * a.inv_t_64 - log_lt;
    const double log_p = ((double)y_p[i] - (double)m_all) * a.inv_t_64 - log_all;
    q_p[i] = exp_of(log_q);
    p_p[i] = exp_of(log_p);
    w_p[i] = (float)(log_p - log_q);
    sum_q += (double)q_p[i];
    kd_64 += (double)above_tangent(q_p[i], p_p[i], w_p[i]);
  });
  sum_q = sum16(sum_q);
  kd_64 = sum16(kd_64);
  const double rest_64 = given && others ? 1.0 - sum_q : 0.0;
  const float rest = rest_64 > 0.0 || rest_64 != rest_64 ? (float)rest_64 : 0.f;
  const float share = others ? exp_of(log_share) : 0.f;                  // the student's of the others
  const float w_rest = rest == 0.f ? 0.f : (float)(log_share - log_64(rest));
  kd_64 += (double)above_tangent(rest, share, w_rest);
  const float over = given ? (float)(sum_q + (double)rest - 1.0) : 0.f;  // where the teacher's entries are more than 1 in all
  const float kd = taught ? (float)(kd_64 + (double)over) : 0.f;
  const float on_kd = taught && weight != 0.f ? weight * a.teacher_slope : 0.f;
  const float on_label = valid && weight != 0.f ? weight * a.label_slope : 0.f;
  const float on_p = on_label + (valid && weight != 0.f ? 2.f * weight * a.z_slope * lse : 0.f);
  __shared__ float sh_loss[kObjRows];
  __shared__ int sh_count[kObjRows];
  if (in && lane == 0) {
    if (a.nll_c) a.nll_c[s] = nll;
    if (a.kd_c) a.kd_c[s] = kd;
    if (a.lse_c) a.lse_c[s] = lse;
    float loss = 0.f;
    if (weight != 0.f) {
      if (valid) loss += weight * (a.label_coef * nll + a.z_coef * lse * lse);
      if (taught) loss += weight * a.teacher_coef * a.temperature * a.temperature * kd;
    }
    const int count = bad_entry || (labelled && !valid) ? -1 : valid || taught ? 1 : 0;
    if (kAll) {
      sh_loss[r] = loss;
      sh_count[r] = count;
    } else {
      a.row_loss_c[s] = make_float2(loss, __builtin_bit_cast(float, count));
    }
  }
  if constexpr (kAll) {
    __syncthreads();
    if (threadIdx.x == 0) {
      double sum = 0.0;
      int n_rows = 0, bad = 0;
      for (int i = 0; i < a.rows; ++i) {
        sum += (double)sh_loss[i];
        n_rows += sh_count[i] > 0;
        bad |= sh_count[i] < 0;
      }
      write_loss(o, sum, n_rows, bad);
    }
  }
  if (!a.rows_c || !in) return;
  // (Q + rest) p - q and (Q + rest) p_rest - rest, whose Q + rest is 1 + over, as q (exp(w) - 1) + over p
  const float kd_others = on_kd == 0.f ? 0.f : on_kd * ((rest == 0.f ? share : share_less(rest, share, w_rest)) + over * share);
  if (lane == 0) {
    ObjRow row;
    ObjRow2 row2 = {__builtin_inff(), 0.f};
    row.label = valid && weight != 0.f ? y : -1;
    row.label_term = on_label;
    if (two) {
      row.base = base;
      row.at = kd_others;
      row2.base = lse;
      row2.at = on_p;
      if (on_p == 0.f) row2.base = __builtin_inff();
    } else if (P) {
      row.base = base;
      row.at = kd_others + on_p * share;
    } else {
      row.base = lse;
      row.at = on_p;
    }
    if (!others || row.at == 0.f) row.base = __builtin_inff(), row.at = 0.f;     // exp2 of -infinity: zeros whatever the logits
    a.rows_c[s] = row;
    if (a.rows2_c) a.rows2_c[s] = row2;
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = lane + 16 * i, v = v_p[i];
    if (e >= a.K) continue;
    float x = 0.f;
    if (v != kNoEntry) {
      if (on_kd != 0.f) x = on_kd * ((q_p[i] == 0.f ? p_p[i] : share_less(q_p[i], p_p[i], w_p[i])) + over * p_p[i]);
      if (on_p != 0.f) x += on_p * expf((y_p[i] - m_all) - log_label);
      if (valid && v == y) x -= on_label;
      if (a.cap > 0.f) x *= Cap(a.cap).slope<false>(z_p[i]);
    }
    a.saved_index_c[at0 + e] = v;
    a.saved_at_c[at0 + e] = x;
  }
}

// From every thread's sum, count and whether an index is out of range (1024 threads), in a fixed order.
__device__ __forceinline__ void reduce_obj_loss(const ObjLoss& o, double a, long long n, int bad) {
  __shared__ double sh[16];
  __shared__ long long sh_n[16];
  __shared__ int sh_bad[16];
  for (int k = 32; k > 0; k >>= 1) {
    a += __shfl_xor(a, k);
    n += __shfl_xor(n, k);
    bad |= __shfl_xor(bad, k);
  }
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) { sh[w] = a; sh_n[w] = n; sh_bad[w] = bad; }
  __syncthreads();
  if (threadIdx.x != 0) return;
  a = 0.0; n = 0; bad = 0;
  for (int i = 0; i < 16; ++i) { a += sh[i]; n += sh_n[i]; bad |= sh_bad[i]; }
  write_loss(o, a, n, bad);
}
// One workgroup, bound by the latency of its loads: sixteen rounds of them at a time.
__global__ __launch_bounds__(1024) void k_obj_loss(const float2* __restrict__ row_loss, long long S, ObjLoss o) {
  double a = 0.0;
  long long n = 0;
  int bad = 0;
  constexpr int kAtOnce = 16;
  for (long long i0 = threadIdx.x; i0 < S; i0 += kAtOnce * 1024) {
    float2 x[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) x[k] = i0 + k * 1024 < S ? row_loss[i0 + k * 1024] : make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int count = __builtin_bit_cast(int, x[k].y);
      a += (double)x[k].x;
      n += count > 0;
      bad |= count < 0;
    }
  }
  reduce_obj_loss(o, a, n, bad);
}

// k_obj_finalize and k_obj_loss of calls without a teacher that are few rows and vocabulary tiles (one_finalizes), from one
// workgroup: up to 16 threads, 2^row_bits apart, have a row and all of its pairs in flight at once, as k_finalize_loss.
constexpr int kOneGroups = 16;
__global__ __launch_bounds__(1024) void k_obj_finalize_one(ObjFinal a, ObjLoss o, int row_bits) {
  __shared__ float2 sh[1024];
  const int s = threadIdx.x & ((1 << row_bits) - 1), g = __builtin_amdgcn_readfirstlane(threadIdx.x >> row_bits), groups = 1024 >> row_bits;
  const bool in = s < a.rows;
  int y = 0;
  float z_y = 0.f, weight = 1.f, m = kMasked, l = 0.f;
  if (in) {
    float2 p[kFinOneTiles];
#pragma unroll
    for (int i = 0; i < kFinOneTiles; ++i) {
      const int vt = g + i * groups;
      p[i] = vt < a.n_vt ? a.part[(size_t)vt * a.part_stride + s] : make_float2(kMasked, 0.f);
    }
    y = a.labels_c[s];
    z_y = a.tgt[s];
    if (a.weights_c) weight = a.weights_c[s];
    fold_lse(m, l, p);
  }
  if (groups > 1) {
    sh[threadIdx.x] = make_float2(m, l);
    __syncthreads();
    if (groups <= 4) {
      for (int i = 1; i < groups; ++i) {
        const float2 q = sh[(threadIdx.x + (i << row_bits)) & 1023];
        merge_lse(m, l, q.x, q.y);
      }
    } else {
      float2 q[kOneGroups];
#pragma unroll
      for (int i = 0; i < kOneGroups; ++i) q[i] = i < groups ? sh[(i << row_bits) | s] : make_float2(kMasked, 0.f);
      m = kMasked;
      l = 0.f;
      fold_lse(m, l, q);
    }
  }
  float loss = 0.f;
  int count = 0;
  if (in && g == 0) {
    const float log_l = logf(l), lse = m + log_l;
    const bool valid = y != a.ignore_index && (unsigned)y < (unsigned)a.V;
    const float nll = valid ? (m - z_y) + log_l : 0.f;
    const bool on = valid && weight != 0.f;
    if (on) loss = weight * (a.label_coef * nll + a.z_coef * lse * lse);
    count = y == a.ignore_index ? 0 : valid ? 1 : -1;
    if (a.nll_c) a.nll_c[s] = nll;
    if (a.lse_c) a.lse_c[s] = lse;
    if (a.rows_c) {
      ObjRow row;
      row.label = on ? y : -1;
      row.label_term = on ? weight * a.label_slope : 0.f;
      row.at = on ? row.label_term + 2.f * weight * a.z_slope * lse : 0.f;
      row.base = row.at == 0.f ? __builtin_inff() : lse;
      a.rows_c[s] = row;
    }
  }
  reduce_obj_loss(o, (double)loss, count > 0, count < 0);
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// Every entry is rounded to bf16, here and in k_obj_entries too, as the matrix instructions of both products take it: dH and dW, themselves
// in bf16, are 2.2e-3 off in place of 1.7e-3, errors of either sign (ObjLoss::unit keeps it so); two bf16 parts an entry would double
// the products, three quarters of a step.
struct ObjGrad {
  const ObjHeader* head;
  const ObjRow* rows;
  const ObjRow2* rows2;              // read where head->two
  const int* index;                  // [rows][K] the teacher's entries and the gradient there, for tiles that put them in themselves
  const float* at;
  int K;                             // 0: none, or k_obj_entries does it
  static constexpr bool kPatch = true;
  // `rows` rows of a tile from row s0 on, kWidth vocabulary entries from v0 on: into the tile at `staged`
  template <int kThreadsOfTile>
  __device__ __forceinline__ void patch(int s0, int n_rows, int v0, int width, int V, char* staged, int row_bytes) const {
    if (!K) return;
    __syncthreads();
    const size_t from = (size_t)s0 * K;
    const FirstEntries first = load_entries<kThreadsOfTile>(index + from, n_rows * K, threadIdx.x);
    each_entry<kThreadsOfTile>(first, index + from, n_rows, K, [&](int r, int k, int v) {
      if ((unsigned)(v - v0) < (unsigned)width && v < V)
        *reinterpret_cast<__bf16*>(staged + r * row_bytes + 2 * (v - v0)) = (__bf16)at[from + (size_t)r * K + k];
    });
  }
  struct Row { ObjRow a; ObjRow2 b; };
  __device__ __forceinline__ Row load(int s) const {
    Row r;
    r.a = rows[s];
    r.b = head->two ? rows2[s] : ObjRow2{0.f, 0.f};
    return r;
  }
  __device__ __forceinline__ Row settle(const Row& r) const { return r; }
  __device__ __forceinline__ int label(const Row& r) const { return r.a.label; }
  __device__ __forceinline__ float label_term(const Row& r, float z) const {
    return head->cap > 0.f ? r.a.label_term * Cap(head->cap).slope<false>(z) : r.a.label_term;
  }
  template <class Top, class F>
  __device__ __forceinline__ void with(const Row& r, Top top, F f) const {
    const float c1 = head->exponent, c2 = head->exponent_label, cap = head->cap;
    if (cap > 0.f) {
      const Cap bend(cap);
      auto capped = [&](auto near) {
        constexpr bool kNear = decltype(near)::value;
        if (head->two)
          f([&](float z) {
            const float y = bend.template y<kNear>(z);
            return bend.template slope<kNear>(z) * (r.a.at * fast_exp2((y - r.a.base) * c1) + r.b.at * fast_exp2((y - r.b.base) * c2));
          });
        else
          f([&](float z) { return bend.template slope<kNear>(z) * (r.a.at * fast_exp2((bend.template y<kNear>(z) - r.a.base) * c1)); });
      };
      if (__any(!bend.near(top()))) capped(std::false_type()); else capped(std::true_type());
    } else if (head->two) {
      f([&](float z) { return r.a.at * fast_exp2((z - r.a.base) * c1) + r.b.at * fast_exp2((z - r.b.base) * c2); });
    } else {
      f([&](float z) { return r.a.at * fast_exp2((z - r.a.base) * c1); });
    }
  }
};

// The teacher's entries of some rows that lie in a window of the vocabulary, into its dlogits.  What bounds it are the scattered stores of
// two bytes: 1.1 million of them, 32768 rows of 256 in one of 7.5 windows, 25 us, also with four entries a thread and 32-bit divisions.
__global__ __launch_bounds__(256) void k_obj_entries(const int* __restrict__ index, const float* __restrict__ at, long long n, int K,
                                                     int v_base, int V, __bf16* __restrict__ G, int ldg) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int v = index[i] - v_base;
  if ((unsigned)v < (unsigned)V) G[(size_t)(i / K) * ldg + v] = (__bf16)at[i];
}

}  // namespace mst
