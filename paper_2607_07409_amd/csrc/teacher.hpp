// A teacher's top entries of a row, as the distillation kernels use them: K <= 256 (id, value) pairs, one per thread of
// a workgroup of 256.  An entry whose id lies outside [0, V) or whose value is -inf (or NaN) is absent.
#pragma once
#include "row_stream.hpp"

namespace dls {

struct TeacherEntry {
  int id;            // -1: absent
  float q, log_q;    // log q natural; q = 0 for an absent entry
};

struct TeacherShared {
  float red[kRowThreads / 64];
};

// sum (or maximum) over the workgroup, in a fixed order, in every thread
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}
__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) v = fmaxf(v, __shfl_xor(v, k));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// This thread's entry of row r, and the row's mass sum_k q_k (1 or 0 where normalised).
__device__ __forceinline__ TeacherEntry teacher_entry(const TeacherArgs& te, int64_t r, int V, TeacherShared& sh,
                                                      float* mass) {
  const int t = threadIdx.x;
  TeacherEntry e = {-1, 0.f, -INFINITY};
  float y = -INFINITY;
  if (t < te.k) {
    const size_t at = (size_t)r * te.k + t;
    e.id = te.ids[at];
    y = te.values[at];
    if (e.id < 0 || e.id >= V || !(y > -INFINITY)) {
      e.id = -1;
      y = -INFINITY;
    }
  }
  if (te.logprobs) {
    e.q = fast_exp2(y * kLog2e);
    e.log_q = y;
    *mass = block_sum(e.q, sh.red);
  } else {
    const float top = block_max(y, sh.red);
    const float d = e.id < 0 ? -INFINITY : (y - top) * te.c;   // (the largest finite values differ by a finite amount)
    const float w = fast_exp2(d);
    const float sum = block_sum(w, sh.red);
    e.q = sum > 0.f ? w / sum : 0.f;
    e.log_q = e.id < 0 ? -INFINITY : (d - fast_log2(sum)) * kLn2;
    *mass = sum > 0.f ? 1.f : 0.f;
  }
  return e;
}

// q (log q - log p) of an entry; log2 of its probability is y - R - l2.  0 for an entry of weight 0.
__device__ __forceinline__ float teacher_term(const TeacherEntry& e, float log2_p) {
  return e.q > 0.f ? e.q * (e.log_q - log2_p * kLn2) : 0.f;
}

}  // namespace dls
