// Distillation of rows of student logits s from a teacher's top entries (id_k, q_k), at temperature T:
//   loss   = sum_k q_k (log q_k - log softmax(s / T)[id_k])
//   d s_v  = g / T (M softmax(s / T)_v - sum_{k: id_k = v} q_k),   M = sum_k q_k, g the row's weight in the total.
//
// The loss needs the row's log-sum-exp, one pass over the logits (row_stream.hpp), and K entries.  Loss and gradient
// together: a row that fits a workgroup's registers is read once and its gradient written from there (k_distill_row);
// others take a second pass that reads an entry and writes one (k_distill_grad, which is also the gradient alone).  The
// teacher's entries of a workgroup's range are written after it, each from its own logit in float32 and rounded once
// (several entries of one id by the first of them).
//
// What bounds it: reads and writes.  2,048 bf16 rows of V = 151,936, loss and gradient in 243 to 257 us: 4.8 to 5.1 TB/s
// of the 1.24 GB read and written, where a large copy reaches 4.93.  The gradient alone of 777 rows of V = 70,001 in
// 55 us (3.9 TB/s), of 900 float32 rows of V = 81,920 in 125 (4.7).  Rows beyond the registers are read twice: 300
// float32 rows of V = 151,936 in 120 us, 3.0 TB/s of what is read once and written (4.5 of what moves).  Small calls are
// latency: 16 rows of V = 32,003, loss and gradient, 9 us of kernel.
#include "teacher.hpp"

namespace dls {

namespace {

constexpr int kThreads = kRowThreads;

struct LossOut {
  float *loss, *lse;   // either may be NULL
  float2* row;         // (R, log2 s; +inf for an empty row) for the gradient pass, or NULL
};

// the loss of a row from its sums, by the whole workgroup
template <typename T>
__device__ __forceinline__ void finish_row(const T* row, int V, int64_t r, const RowSum& a, const TeacherArgs& te,
                                           TeacherShared<kThreads>& sh, const LossOut& o) {
  float mass;
  const TeacherEntry e = teacher_entry<kThreads>(te, teacher_raw(te, r, V), sh, &mass);
  const float l2 = a.s == 0.f ? INFINITY : fast_log2(a.s);
  const float x = e.id >= 0 ? to_f32(row[e.id]) : -INFINITY;
  const float loss = block_sum<kThreads>(teacher_term(e, above_ref(x, te.c, a.R) - l2), sh.red);
  if (threadIdx.x == 0) {
    if (o.loss) o.loss[r] = loss;
    if (o.lse) o.lse[r] = row_lse(a);
    if (o.row) o.row[r] = make_float2(a.R, l2);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_distill_part(const T* __restrict__ L, int V, int64_t stride, TeacherArgs te,
                                                           float2* __restrict__ part_sums, LossOut o) {
  constexpr int N = Chunk<T>::N;
  __shared__ RowShared<> shr;
  __shared__ TeacherShared<kThreads> sht;
  const int part = blockIdx.y, parts = gridDim.y;
  const int64_t r = blockIdx.x;
  const T* row = L + (size_t)r * stride;
  const RowRange g = row_range(row, V, part, parts);
  RowSum a = row_empty();
  row_edges(g, V, part, parts, [&](int v) {
    const float x = to_f32(row[v]);
    row_fold<1, false>(a, &x, x, te.c);
  });
  row_chunks<2>(   // (four loads a thread in flight are slower: 2,048 rows of V = 32,003 in 31.0 us, with two 28.6)
      row, g,
      [&](const uint4* raw, auto n, int) {
        float x[N * n];
#pragma unroll
        for (int u = 0; u < n; ++u) Chunk<T>::widen(raw[u], x + u * N);
        row_fold<N * n, false>(a, x, max_of<N * n>(x), te.c);
      },
      [](int) {});
  a = row_block_merge<false>(a, shr);
  if (parts == 1) finish_row(row, V, r, a, te, sht, o);
  else if (threadIdx.x == 0) part_sums[(size_t)r * parts + part] = make_float2(a.R, a.s);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_distill_finish(const T* __restrict__ L, int V, int64_t stride,
                                                             TeacherArgs te, int parts,
                                                             const float2* __restrict__ part_sums, LossOut o) {
  __shared__ RowShared<> shr;
  __shared__ TeacherShared<kThreads> sht;
  const int64_t r = blockIdx.x;
  RowSum a = row_empty();
  if ((int)threadIdx.x < parts) {   // parts <= 256
    const float2 p = part_sums[(size_t)r * parts + threadIdx.x];
    a.R = p.x;
    a.s = p.y;
  }
  a = row_block_merge<false>(a, shr);
  finish_row(L + (size_t)r * stride, V, r, a, te, sht, o);
}

// 16-byte stores at any element alignment (the gradient's rows may be aligned otherwise than the logits')
template <typename T> struct Store;
template <> struct Store<float> {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  __device__ __forceinline__ static void chunk(float* p, const float* v) {
    vec o = {v[0], v[1], v[2], v[3]};
    __builtin_nontemporal_store(o, reinterpret_cast<vec*>(p));
  }
  __device__ __forceinline__ static void one(float* p, float v) { *p = v; }
};
template <> struct Store<bf16_t> {
  typedef __bf16 vec __attribute__((ext_vector_type(8)));
  typedef float vecf __attribute__((ext_vector_type(8)));
  typedef unsigned words __attribute__((ext_vector_type(4), aligned(2)));
  __device__ __forceinline__ static void chunk(bf16_t* p, const float* v) {
    const vecf f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    __builtin_nontemporal_store(__builtin_bit_cast(words, __builtin_convertvector(f, vec)), reinterpret_cast<words*>(p));
  }
  __device__ __forceinline__ static void one(bf16_t* p, float v) { *p = __builtin_bit_cast(bf16_t, (__bf16)v); }
};

// The dense part of a gradient, f 2^(y - R), of n entries; 0 where f is, whatever the entries.  R and f are the same in
// every lane of the workgroup, so the choice is a scalar branch; a clamped R holds no difference of the size of a logarithm,
// so there a probability is at most 1.
struct Dense {
  float c, R, f;
  bool plain;
  __device__ __forceinline__ Dense(float c, float R_, float f_) : c(c) {
    R = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(R_)));
    f = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(f_)));
    plain = fabsf(R) < kPlainRef && f != 0.f;
  }
  template <int n>
  __device__ __forceinline__ void operator()(const float* x, float* d) const {
    if (plain) {
#pragma unroll
      for (int i = 0; i < n; ++i) d[i] = f * fast_exp2(__builtin_fmaf(x[i], c, -R));
    } else if (f != 0.f) {
#pragma unroll
      for (int i = 0; i < n; ++i) d[i] = f * fast_exp2(fminf(above_ref(x[i], c, R), 0.f));
    } else {
#pragma unroll
      for (int i = 0; i < n; ++i) d[i] = 0.f;
    }
  }
  __device__ __forceinline__ float operator()(float x) const {
    float d;
    operator()<1>(&x, &d);
    return d;
  }
};

// Loss and gradient with the row on chip: a workgroup of NT threads reads its row once, NCH 16-byte pieces a thread,
// into registers, and writes the gradient from there.  All of a row's loads are in flight together.
template <typename T, int NT, int NCH>
__global__ __launch_bounds__(NT) void k_distill_row(const T* L, int V, int64_t stride, TeacherArgs te,
                                                    const float* __restrict__ weight, LossOut o, T* G, int64_t gstride) {
  constexpr int N = Chunk<T>::N;
  __shared__ RowShared<NT> shr;
  __shared__ TeacherShared<NT> sht;
  __shared__ int ids[256];
  __shared__ float qs[256];
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x;
  const T* row = L + (size_t)r * stride;
  T* out = G + (size_t)r * gstride;
  const RowRange g = row_range(row, V, 0, 1);
  // (one address for the row and 32-bit offsets: the registers are needed for the row itself)
  const char* from = reinterpret_cast<const char*>(row + g.h0);
  char* to = reinterpret_cast<char*>(out + g.h0);
  uint4 raw[NCH];
  if (g.c1 > 0) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) raw[i] = stream_load16(from + (uint32_t)min(t + i * NT, g.c1 - 1) * 16u);
  }
  const TeacherRaw tr = teacher_raw(te, r, V);
  const float xk = tr.id >= 0 ? to_f32(row[tr.id]) : -INFINITY;   // read before anything is written: G may be L
  RowSum a = row_empty();
  float edge[2] = {0.f, 0.f};   // this thread's entry before the first piece, and behind the last
  const bool has[2] = {t < g.h0, t < V - g.tail0};
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (has[e]) {
      edge[e] = to_f32(row[e == 0 ? t : g.tail0 + t]);
      row_fold<1, false>(a, &edge[e], edge[e], te.c);
    }
#pragma unroll
  for (int i = 0; i < NCH; ++i)
    if (t + i * NT < g.c1) {
      float x[N];
      Chunk<T>::widen(raw[i], x);
      row_fold<N, false>(a, x, max_of<N>(x), te.c);
    }
  a = row_block_merge<false>(a, shr);
  float mass;
  const TeacherEntry e = teacher_entry<NT>(te, tr, sht, &mass);
  if (t < 256) {
    ids[t] = e.id;
    qs[t] = e.q;
  }
  const float l2 = a.s == 0.f ? INFINITY : fast_log2(a.s);
  const float loss = block_sum<NT>(teacher_term(e, above_ref(xk, te.c, a.R) - l2), sht.red);   // (its barriers cover ids, qs)
  if (t == 0) {
    if (o.loss) o.loss[r] = loss;
    if (o.lse) o.lse[r] = row_lse(a);
  }
  const float w = (weight ? weight[r] : 1.f) * te.inv_temp, f = a.s == 0.f || mass == 0.f ? 0.f : w * mass / a.s;
  const Dense dense(te.c, a.R, f);
  bool mine = e.id >= 0;
  float entry = 0.f;
  if (mine) {
    float q = 0.f;
    for (int j = 0; j < te.k; ++j) {
      const bool same = ids[j] == e.id;
      q += same ? qs[j] : 0.f;
      mine = mine && !(same && j < t);
    }
    entry = dense(xk) - w * q;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (has[e]) Store<T>::one(out + (e == 0 ? t : g.tail0 + t), dense(edge[e]));
#pragma unroll
  for (int i = 0; i < NCH; ++i)
    if (t + i * NT < g.c1) {
      float x[N], d[N];
      Chunk<T>::widen(raw[i], x);
      dense.template operator()<N>(x, d);
      Store<T>::chunk(reinterpret_cast<T*>(to + (uint32_t)(t + i * NT) * 16u), d);
    }
  __syncthreads();   // the row is written before its teacher entries are
  if (mine) Store<T>::one(out + e.id, entry);
}

// The gradient of a part of a row, at most kGradPieces 16-byte pieces a thread, whose loads are all on their way before
// the teacher's entries are looked at.  The row's sums come from the loss pass, or from its log-sum-exp.
constexpr int kGradPieces = 10;
template <typename T>
__global__ __launch_bounds__(kThreads) void k_distill_grad(const T* L, int V, int64_t stride, TeacherArgs te,
                                                           const float* __restrict__ lse,
                                                           const float2* __restrict__ row_stats,
                                                           const float* __restrict__ weight, T* G, int64_t gstride) {
  constexpr int N = Chunk<T>::N;
  __shared__ TeacherShared<kThreads> sht;
  __shared__ int ids[kThreads];
  __shared__ float qs[kThreads];
  const int part = blockIdx.y, parts = gridDim.y, t = threadIdx.x;
  const int64_t r = blockIdx.x;
  const T* row = L + (size_t)r * stride;
  T* out = G + (size_t)r * gstride;
  const RowRange g = row_range(row, V, part, parts);
  uint4 raw[kGradPieces];
  if (g.c1 > g.c0) {
#pragma unroll
    for (int i = 0; i < kGradPieces; ++i)
      raw[i] = stream_load16(row + g.h0 + (size_t)min(g.c0 + t + i * kThreads, g.c1 - 1) * N);
  }
  const TeacherRaw tr = teacher_raw(te, r, V);
  // my entry, where its id lies in this part's range: read before anything is written, G may be L
  const int lo = part == 0 ? 0 : g.h0 + g.c0 * N, hi = part == parts - 1 ? V : g.h0 + g.c1 * N;
  bool mine = tr.id >= lo && tr.id < hi;
  const float xk = mine ? to_f32(row[tr.id]) : 0.f;
  float edge[2] = {0.f, 0.f};   // this thread's entry before the row's first piece, and behind its last
  const bool has[2] = {part == 0 && t < g.h0, part == parts - 1 && t < V - g.tail0};
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (has[e]) edge[e] = to_f32(row[e == 0 ? t : g.tail0 + t]);
  // softmax(s / T)_v = 2^(y - R) f
  float R, f;
  if (row_stats) {
    const float2 p = row_stats[r];
    R = p.x;
    f = fast_exp2(-p.y);
  } else {
    // lse log2(e) to twice the precision: the part that R cannot hold goes into the factor
    const float l = lse[r];
    R = __builtin_amdgcn_fmed3f(l * kLog2e, -kMostY, kMostY);
    f = l == -INFINITY ? 0.f
        : !(l < INFINITY) ? __builtin_nanf("")
        : fabsf(R) < kPlainRef ? fast_exp2(-(__builtin_fmaf(l, kLog2e, -R) + l * kLog2eLow)) : 1.f;
  }
  const float w = (weight ? weight[r] : 1.f) * te.inv_temp;
  float mass;
  const TeacherEntry e = teacher_entry<kThreads>(te, tr, sht, &mass);
  ids[t] = e.id;
  qs[t] = e.q;
  __syncthreads();   // (also: every entry of the teacher's has been read)
  const Dense dense(te.c, R, mass == 0.f ? 0.f : w * mass * f);
  float entry = 0.f;
  if (mine) {   // several entries of one id are the first one's
    float q = 0.f;
    for (int j = 0; j < te.k; ++j) {
      const bool same = ids[j] == e.id;
      q += same ? qs[j] : 0.f;
      mine = mine && !(same && j < t);
    }
    entry = dense(xk) - w * q;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (has[e]) Store<T>::one(out + (e == 0 ? t : g.tail0 + t), dense(edge[e]));
#pragma unroll
  for (int i = 0; i < kGradPieces; ++i) {
    const int c = g.c0 + t + i * kThreads;
    if (c < g.c1) {
      float x[N], d[N];
      Chunk<T>::widen(raw[i], x);
      dense.template operator()<N>(x, d);
      Store<T>::chunk(out + g.h0 + (size_t)c * N, d);
    }
  }
  __syncthreads();   // the part is written before its teacher entries are
  if (mine) Store<T>::one(out + e.id, entry);
}

// workgroups per row of the gradient pass: as many as its pieces need, more where rows are few
int grad_parts(int64_t rows, int32_t V, int elem_bytes) {
  const int64_t few = row_parts(rows, V, elem_bytes), per = (int64_t)kThreads * kGradPieces * (16 / elem_bytes);
  return (int)std::max<int64_t>(1, std::max<int64_t>(few, (V + per - 1) / per));
}

template <typename T>
hipError_t launch_grad_t(const DistillArgs& a, const float2* row_stats, hipStream_t st) {
  const dim3 grid((unsigned)a.rows, (unsigned)grad_parts(a.rows, a.V, (int)sizeof(T)));
  k_distill_grad<T><<<grid, kThreads, 0, st>>>((const T*)a.logits, a.V, a.stride, a.teacher, a.lse, row_stats, a.weight,
                                               (T*)a.grad, a.grad_stride);
  return hipGetLastError();
}

// A row whose pieces fit a workgroup's registers is read once, else twice, by the loss's kernels and k_distill_grad (700
// rows of V = 32,003: 25 us and 37; 2,048 of V = 151,936: 254 and 376).  By 1,024 threads, the least work for each; from
// 512 rows on (two a CU) short ones by 256, so that several rows are in flight on a CU (V = 16,001: 1,100 rows in 22.7 us,
// with 1,024 threads 34; 1,500 rows of V = 24,001 37 and 44).
template <typename T, int NT, int NCH>
hipError_t launch_row_t(const DistillArgs& a, hipStream_t st) {
  const LossOut o = {a.out_loss, a.out_lse, nullptr};
  k_distill_row<T, NT, NCH><<<(unsigned)a.rows, NT, 0, st>>>((const T*)a.logits, a.V, a.stride, a.teacher, a.weight, o,
                                                             (T*)a.grad, a.grad_stride);
  return hipGetLastError();
}
template <typename T>
bool row_fits(int64_t rows, int32_t V) {
  // (few long rows: split over the card they are done sooner, also if read twice; 64 bf16 rows of V = 151,936 in 21.4 us,
  // by a workgroup each 24.9; of V = 100,003 20.3 and 20.5, of 70,001 20.2 and 16.8; 128 of V = 151,936 28.4 and 25.6)
  if (rows <= 64 && V > 100000) return false;
  return V <= 1024 * 20 * Chunk<T>::N;
}
template <typename T>
hipError_t launch_row(const DistillArgs& a, hipStream_t st) {
  const int64_t pieces = (a.V + Chunk<T>::N - 1) / Chunk<T>::N;
  if (a.rows >= 512 && pieces <= 256 * 12) return launch_row_t<T, 256, 12>(a, st);
  return pieces <= 1024 * 5    ? launch_row_t<T, 1024, 5>(a, st)
         : pieces <= 1024 * 10 ? launch_row_t<T, 1024, 10>(a, st)
                               : launch_row_t<T, 1024, 20>(a, st);
}

template <typename T>
hipError_t launch_loss_t(const DistillArgs& a, hipStream_t st) {
  if (a.grad && row_fits<T>(a.rows, a.V)) return launch_row<T>(a, st);
  const int parts = row_parts(a.rows, a.V, (int)sizeof(T));
  float2* rows = (float2*)a.ws;
  float2* sums = rows + a.rows;
  const LossOut o = {a.out_loss, a.out_lse, a.grad ? rows : nullptr};
  const T* L = (const T*)a.logits;
  k_distill_part<T><<<dim3((unsigned)a.rows, (unsigned)parts), kThreads, 0, st>>>(L, a.V, a.stride, a.teacher, sums, o);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (parts > 1) {
    k_distill_finish<T><<<(unsigned)a.rows, kThreads, 0, st>>>(L, a.V, a.stride, a.teacher, parts, sums, o);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return a.grad ? launch_grad_t<T>(a, rows, st) : hipSuccess;
}

}  // namespace

size_t distill_workspace_bytes(int64_t rows, int32_t V) {
  // the larger of the two types' needs: the float32 rows split further
  const int parts = row_parts(rows, V, 4);
  return (size_t)rows * sizeof(float2) * (1 + (parts > 1 ? parts : 0));
}

hipError_t launch_distill_loss(const DistillArgs& a, hipStream_t st) {
  return a.dtype == DLS_BF16 ? launch_loss_t<bf16_t>(a, st) : launch_loss_t<float>(a, st);
}

hipError_t launch_distill_grad(const DistillArgs& a, hipStream_t st) {
  return a.dtype == DLS_BF16 ? launch_grad_t<bf16_t>(a, nullptr, st) : launch_grad_t<float>(a, nullptr, st);
}

}  // namespace dls
