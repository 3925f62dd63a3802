// One pass over rows of logits: what the log-probability and distillation kernels share.
//
// A row of V entries is split into `parts` contiguous ranges, one workgroup each (of 256 threads here; distillation with
// its gradient also takes whole rows by 1,024).  A thread reads 16-byte chunks (coalesced over the workgroup; in row_chunks
// the next U are in flight while U are folded) and keeps, for y = x c with c = log2(e) / T,
//   R   the reference: a y that was the largest when it was taken, and is within kLazy of the largest so far,
//   s   sum 2^(y - R),   and where the entropy is wanted   t = sum 2^(y - R) (y - R),
// all in float32, so that log-sum-exp = ln2 (R + log2 s), log p = ln2 (y - R - log2 s) and H = ln2 (log2 s - t / s).
// One fused multiply-add forms y - R with a single rounding, whatever the size of R.
#pragma once
#include <type_traits>

#include "dels_internal.hpp"
#include "stream_load.hpp"

namespace dls {

constexpr int kRowThreads = 256;
constexpr float kNoRef = -2.0e38f;        // R before the first entry (finite: no inf - inf)
constexpr float kPlainRef = 0x1p80f;      // |R| below this: y - R is formed by one fma
constexpr float kMostY = 1.0e38f;         // entries beyond it count as it (only where no entry of the row is plain)
constexpr float kLog2eLow = 1.92596299e-8f;   // log2(e) - kLog2e
constexpr float kNoTerm = -1500.f;        // 2^kNoTerm = 0: a lower exponent adds nothing to s or t

// Reductions over groups of W lanes (a power of two), in a fixed order, the result in every lane: by lane permutations of
// the vector unit, not through the LDS
template <int W, typename Op>
__device__ __forceinline__ float lanes_reduce(float v, Op op) {
  auto dpp = [&](auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if constexpr (W >= 2) v = op(v, dpp(std::integral_constant<int, 0xB1>{}));     // lane ^ 1
  if constexpr (W >= 4) v = op(v, dpp(std::integral_constant<int, 0x4E>{}));     // lane ^ 2
  if constexpr (W >= 8) v = op(v, dpp(std::integral_constant<int, 0x141>{}));    // the other half of eight
  if constexpr (W >= 16) v = op(v, dpp(std::integral_constant<int, 0x140>{}));   // the other half of sixteen
  if constexpr (W >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  if constexpr (W >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  return v;
}
template <int W = 64>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_reduce<W>(v, [](float a, float b) { return a + b; });
}
template <int W = 64>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_reduce<W>(v, [](float a, float b) { return fmaxf(a, b); });
}

struct RowSum {
  float R, s, t;
};
__device__ __forceinline__ RowSum row_empty() { return {kNoRef, 0.f, 0.f}; }

// y - R of one entry; -inf for a masked one.  Rows whose largest entries lie beyond kPlainRef (a row of the
// type's lowest value, say) take the entries' products clamped, so that nothing overflows.  NaN stays NaN, and +inf
// (always here, since it takes R there) becomes NaN, so that such a row's sum is NaN and all that comes of it.
__device__ __forceinline__ float above_ref(float x, float c, float R) {
  if (fabsf(R) < kPlainRef) return __builtin_fmaf(x, c, -R);
  return x == -INFINITY ? -INFINITY : __builtin_fmaf(x, 0.f, __builtin_amdgcn_fmed3f(x * c, -kMostY, kMostY) - R);
}

template <bool ENT>
__device__ __forceinline__ void row_rescale(RowSum& a, float R) {
  const float d = fmaxf(a.R - R, kNoTerm), r = fast_exp2(d);
  if (ENT) a.t = r * __builtin_fmaf(a.s, d, a.t);
  a.s *= r;
  a.R = R;
}

// The reference moves only where an entry passes it by kLazy, so that after a row's first entries hardly any wave
// rescales: exponentials of up to 2^kLazy are as exact as others.
constexpr float kLazy = 8.f;

template <int n, bool ENT>
__device__ __forceinline__ void row_add(RowSum& a, const float* x, float c) {
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const float y = __builtin_fmaf(x[i], c, -a.R);   // -inf for a masked entry
    const float e = fast_exp2(y);
    a.s += e;
    if (ENT) a.t = __builtin_fmaf(e, fmaxf(y, kNoTerm), a.t);
  }
}
// the same where the reference moves, or is none yet, or lies far from any logit
template <int n, bool ENT>
__device__ __forceinline__ void row_add_moved(RowSum& a, const float* x, float cm, float c) {
  if (cm > -INFINITY) row_rescale<ENT>(a, fmaxf(a.R, __builtin_amdgcn_fmed3f(cm * c, -kMostY, kMostY)));
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const float y = above_ref(x[i], c, a.R), e = fast_exp2(y);
    a.s += e;
    if (ENT) a.t = __builtin_fmaf(e, fmaxf(y, kNoTerm), a.t);
  }
}
// n entries whose largest is cm
template <int n, bool ENT>
__device__ __forceinline__ void row_fold(RowSum& a, const float* x, float cm, float c) {
  const bool move = cm * c > a.R + kLazy || a.R < -kPlainRef;
  if (__builtin_amdgcn_ballot_w64(move) && move) {
    row_add_moved<n, ENT>(a, x, cm, c);
    return;
  }
  row_add<n, ENT>(a, x, c);
}

template <bool ENT>
__device__ __forceinline__ RowSum row_merge(RowSum a, RowSum b) {
  const float R = fmaxf(a.R, b.R);
  row_rescale<ENT>(a, R);
  row_rescale<ENT>(b, R);
  return {R, a.s + b.s, ENT ? a.t + b.t : 0.f};
}

// over groups of W lanes, the same in every lane: the largest reference first, then one rescale and a sum
template <bool ENT, int W = 64>
__device__ __forceinline__ RowSum row_wave_merge(RowSum a) {
  row_rescale<ENT>(a, lanes_max<W>(a.R));
  a.s = lanes_sum<W>(a.s);
  if (ENT) a.t = lanes_sum<W>(a.t);
  return a;
}

// over a workgroup of NT threads, in a fixed order; every thread gets the total
template <int NT = kRowThreads>
struct RowShared {
  float R[NT / 64], s[NT / 64], t[NT / 64];
};
template <bool ENT, int NT>
__device__ __forceinline__ RowSum row_block_merge(RowSum a, RowShared<NT>& sh) {
  a = row_wave_merge<ENT>(a);
  const int wave = threadIdx.x >> 6, from = threadIdx.x % (NT / 64);
  if ((threadIdx.x & 63) == 0) {
    sh.R[wave] = a.R;
    sh.s[wave] = a.s;
    if (ENT) sh.t[wave] = a.t;
  }
  __syncthreads();
  return row_wave_merge<ENT, NT / 64>(RowSum{sh.R[from], sh.s[from], ENT ? sh.t[from] : 0.f});
}

// natural log-sum-exp; -inf for a row without an entry above -inf (whose sum is 0: NaN is not)
__device__ __forceinline__ float row_lse(const RowSum& a) {
  return a.s == 0.f ? -INFINITY : (a.R + fast_log2(a.s)) * kLn2;
}

// entries before the row's first 16-byte boundary
template <typename T>
__device__ __forceinline__ int row_head(const T* p, int V) {
  const int h = (int)(((16u - ((uint32_t)(uintptr_t)p & 15u)) & 15u) / sizeof(T));
  return h < V ? h : V;
}

// the part of a row that a workgroup reads: chunks [c0, c1), entry h0 + c N first in chunk c; the first part has
// the row's h0 head entries as well, the last one the entries from tail0 on
struct RowRange {
  int h0, c0, c1, tail0;
};
template <typename T>
__device__ __forceinline__ RowRange row_range(const T* row, int V, int part, int parts) {
  constexpr int N = Chunk<T>::N;
  RowRange r;
  r.h0 = row_head(row, V);
  const int nch = (V - r.h0) / N;
  r.tail0 = r.h0 + nch * N;
  r.c0 = (int)((int64_t)nch * part / parts);
  r.c1 = (int)((int64_t)nch * (part + 1) / parts);
  return r;
}
// the head and tail entries of this part: f(index) by the thread that has one
template <typename F>
__device__ __forceinline__ void row_edges(const RowRange& r, int V, int part, int parts, F f) {
  const int t = threadIdx.x;
  if (part == 0 && t < r.h0) f(t);
  if (part == parts - 1 && t < V - r.tail0) f(r.tail0 + t);
}

// (as an instruction: the compiler would first pass every loaded value through a maximum of its own, for signalling NaN)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}
template <int n>
__device__ __forceinline__ float max_of(const float* x) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i + 1 < n; i += 2) m = max3(m, x[i], x[i + 1]);
  return n % 2 ? m : max3(m, x[n - 1], x[n - 1]);
}

// Every chunk of the range, in iterations of U chunks a thread: eight lanes have the 8 U chunks of one block, 128 bytes
// of it at a load, so that a block is one stretch of memory and the blocks, numbered iteration by iteration, rise
// along the row.  `fold(raw, n, u)` gets n chunks at a time, the iteration's u-th first: U in every whole iteration,
// single ones in the last; `pass(iteration)` comes after each.  Loads run an iteration ahead (chunks past the range clamped to its last: loaded,
// never folded).
constexpr int kBlockLanes = 8;
template <int U, typename T, typename Fold, typename Pass>
__device__ __forceinline__ void row_chunks(const T* row, const RowRange& r, Fold fold, Pass pass) {
  constexpr int NT = kRowThreads;
  if (r.c1 <= r.c0) return;
  const int t = threadIdx.x, mine = r.c0 + t / kBlockLanes * (kBlockLanes * U) + t % kBlockLanes;
  const char* base = reinterpret_cast<const char*>(row + r.h0);   // one address, 32-bit offsets (a row is below 2^26 bytes)
  const uint32_t last = (uint32_t)(r.c1 - 1) * 16;
  uint32_t off = (uint32_t)mine * 16;
  uint4 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) raw[u] = stream_load16(base + min(off + u * kBlockLanes * 16, last));
  int it = 0;
  for (int b = r.c0; b < r.c1; b += NT * U, ++it) {
    uint4 next[U];
    off += U * NT * 16;
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = stream_load16(base + min(off + u * kBlockLanes * 16, last));
    if (b + NT * U <= r.c1) {
      fold(raw, std::integral_constant<int, U>{}, 0);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (mine + (b - r.c0) + u * kBlockLanes < r.c1) fold(raw + u, std::integral_constant<int, 1>{}, u);
    }
    pass(it);
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = next[u];
  }
}

// workgroups per row: about four per CU when rows are few, each range at least two chunks a thread
inline int row_parts(int64_t rows, int32_t V, int elem_bytes) {
  const int64_t p = (1024 + rows - 1) / std::max<int64_t>(rows, 1);
  const int64_t cap = V / (kRowThreads * 2 * (16 / elem_bytes));
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(p, cap), 256));
}

}  // namespace dls
