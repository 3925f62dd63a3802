// A teacher's top entries of a row, as the distillation kernels use them: K <= 256 (id, value) pairs, one per thread of
// a workgroup of 256 threads or more.  An entry whose id lies outside [0, V) or whose value is -inf is absent.
#pragma once
#include "row_stream.hpp"

namespace dls {

struct TeacherEntry {
  int id;            // -1: absent
  float q, log_q;    // log q natural; q = 0 for an absent entry
};

template <int NT>
struct TeacherShared {
  float red[NT / 64];
};

// sum (or maximum) over a workgroup of NT threads, in a fixed order, in every thread
template <int NT>
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = lanes_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return lanes_sum<NT / 64>(red[threadIdx.x % (NT / 64)]);
}
template <int NT>
__device__ __forceinline__ float block_max(float v, float* red) {
  v = lanes_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return lanes_max<NT / 64>(red[threadIdx.x % (NT / 64)]);
}

// This thread's entry of row r as it is stored: id -1 and -inf for an absent one.
struct TeacherRaw {
  int id;
  float y;
};
__device__ __forceinline__ TeacherRaw teacher_raw(const TeacherArgs& te, int64_t r, int V) {
  TeacherRaw e = {-1, -INFINITY};
  if ((int)threadIdx.x < te.k) {
    const size_t at = (size_t)r * te.k + threadIdx.x;
    e.id = te.ids[at];
    e.y = te.values[at];
    if (e.id < 0 || e.id >= V || e.y == -INFINITY) e = TeacherRaw{-1, -INFINITY};
  }
  return e;
}
// This thread's entry, and the row's mass sum_k q_k (where normalised 1, 0 without entries, or NaN as the values are).
template <int NT>
__device__ __forceinline__ TeacherEntry teacher_entry(const TeacherArgs& te, TeacherRaw raw, TeacherShared<NT>& sh,
                                                      float* mass) {
  TeacherEntry e = {raw.id, 0.f, -INFINITY};
  if (te.logprobs) {
    e.q = fast_exp2(raw.y * kLog2e);
    e.log_q = raw.y;
    *mass = block_sum<NT>(e.q, sh.red);
  } else {
    const float top = block_max<NT>(raw.y, sh.red);
    const float d = e.id < 0 ? -INFINITY : (raw.y - top) * te.c;   // (the largest finite values differ by a finite amount)
    const float w = fast_exp2(d);
    const float sum = block_sum<NT>(w, sh.red);
    e.q = sum == 0.f ? 0.f : w / sum;
    e.log_q = e.id < 0 ? -INFINITY : (d - fast_log2(sum)) * kLn2;
    *mass = sum == 0.f ? 0.f : sum / sum;
  }
  return e;
}

// q (log q - log p) of an entry; log2 of its probability is y - R - l2.  0 for an entry of weight 0.
__device__ __forceinline__ float teacher_term(const TeacherEntry& e, float log2_p) {
  return e.q == 0.f ? 0.f : e.q * (e.log_q - log2_p * kLn2);
}

}  // namespace dls
