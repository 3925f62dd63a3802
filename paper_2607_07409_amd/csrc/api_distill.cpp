// C ABI of the operators that score tokens and teach a local head: argument checks (host only, before any HIP
// call), workspace sizing and dispatch.
#include <hip/hip_runtime.h>

#include <cmath>

#include "api_util.hpp"
#include "dels_internal.hpp"

using namespace dls::abi;

namespace {

constexpr int64_t kMostRows = 1 << 20;
constexpr int32_t kMostV = 1 << 24;
constexpr int32_t kMostK = 256;

bool size_ok(int64_t rows, int32_t V) { return rows > 0 && rows <= kMostRows && V > 0 && V <= kMostV; }

dls_status check_rows(int64_t rows, int32_t V) {
  if (rows < 0 || rows > kMostRows) return fail(DLS_ERR_SHAPE, "rows=%lld outside [0, 2^20]", (long long)rows);
  if (V < 1 || V > kMostV) return fail(DLS_ERR_SHAPE, "V=%d outside [1, 2^24]", V);
  return DLS_OK;
}

dls_status check_stride(int64_t stride, int32_t V, const char* name) {
  if (stride < V || stride > ((int64_t)1 << 40))
    return fail(DLS_ERR_SHAPE, "%s=%lld must lie in [V, 2^40]", name, (long long)stride);
  return DLS_OK;
}

dls_status check_temperature(float t) {
  if (!(t >= 1e-4f && t <= 1e4f)) return fail(DLS_ERR_ARG, "temperature %g outside [1e-4, 1e4]", (double)t);
  return DLS_OK;
}

dls_status check_teacher(const dls_teacher& t) {
  if (t.k < 1 || t.k > kMostK) return fail(DLS_ERR_SHAPE, "teacher.k=%d outside [1, 256]", t.k);
  if (t.flags & ~DLS_TEACHER_LOGPROBS) return fail(DLS_ERR_ARG, "unknown teacher flags 0x%x", t.flags);
  if (t.reserved != 0) return fail(DLS_ERR_ARG, "teacher.reserved must be 0");
  return check_temperature(t.temperature);
}

dls_status check_teacher_pointers(const dls_teacher& t) {
  if (!t.ids || !t.values) return fail(DLS_ERR_ARG, "teacher.ids or teacher.values is NULL");
  if (!aligned(t.ids, 4) || !aligned(t.values, 4)) return fail(DLS_ERR_ARG, "teacher.ids or teacher.values is misaligned");
  return DLS_OK;
}

dls_status check_head_sizes(int32_t V, int32_t r) {
  if (V < 1 || V > dls::kHeadMostV) return fail(DLS_ERR_SHAPE, "V=%d outside [1, 2^20]", V);
  if (r < 8 || r > 256 || r % 8) return fail(DLS_ERR_SHAPE, "r=%d must be a multiple of 8 in [8, 256]", r);
  return DLS_OK;
}

dls::TeacherArgs teacher_args(const dls_teacher& t) {
  return {t.ids, t.values, t.k, (t.flags & DLS_TEACHER_LOGPROBS) ? 1 : 0, (float)(1.4426950408889634 / (double)t.temperature),
          1.f / t.temperature};
}

dls_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (bytes < need) return fail(DLS_ERR_WORKSPACE, "workspace %zu bytes < %zu required", bytes, need);
  if (need && (!ws || !aligned(ws, 16))) return fail(DLS_ERR_ARG, "workspace is NULL or not 16-byte aligned");
  return DLS_OK;
}

size_t elem(int dtype) { return dtype == DLS_BF16 ? 2 : 4; }

}  // namespace

extern "C" {

size_t dls_token_logprobs_workspace_size(int64_t rows, int32_t V, int32_t top_k) {
  if (!size_ok(rows, V) || top_k < 0 || top_k > kMostK) return 0;
  return std::max(dls::logprobs_layout(rows, V, 4, top_k).total, dls::logprobs_layout(rows, V, 2, top_k).total);
}

dls_status dls_token_logprobs(const void* logits, dls_dtype dtype_in, int64_t rows, int32_t V, int64_t row_stride,
                              const int32_t* tokens, float temperature, int32_t top_k, dls_token_stats* out_stats,
                              int32_t* out_top_ids, float* out_top_logprobs, void* workspace, size_t ws_bytes,
                              void* stream) {
  clear_error();
  const int dtype = enum_bits(dtype_in);
  dls_status s;
  if (!valid_dtype(dtype)) return fail(DLS_ERR_DTYPE, "unknown dtype %d", dtype);
  if ((s = check_rows(rows, V)) != DLS_OK || (s = check_stride(row_stride, V, "row_stride")) != DLS_OK) return s;
  if (top_k < 0 || top_k > kMostK) return fail(DLS_ERR_SHAPE, "top_k=%d outside [0, 256]", top_k);
  if ((s = check_temperature(temperature)) != DLS_OK) return s;
  if (rows == 0) return DLS_OK;
  if (!logits || !out_stats || (top_k > 0 && (!out_top_ids || !out_top_logprobs)))
    return fail(DLS_ERR_ARG, "required pointer is NULL");
  if (!aligned(logits, elem(dtype)) || !aligned(out_stats, 4) || !aligned(tokens, 4) || !aligned(out_top_ids, 4) ||
      !aligned(out_top_logprobs, 4))
    return fail(DLS_ERR_ARG, "misaligned pointer");
  if ((s = check_workspace(workspace, ws_bytes, dls_token_logprobs_workspace_size(rows, V, top_k))) != DLS_OK) return s;
  if ((s = check_device()) != DLS_OK) return s;
  dls::LogprobsArgs a;
  a.logits = logits;
  a.dtype = static_cast<dls_dtype>(dtype);
  a.rows = rows;
  a.V = V;
  a.stride = row_stride;
  a.tokens = tokens;
  a.temperature = temperature;
  a.k = top_k;
  a.out = out_stats;
  a.top_ids = out_top_ids;
  a.top_logprobs = out_top_logprobs;
  a.ws = (char*)workspace;
  const hipError_t e = dls::launch_logprobs(a, (hipStream_t)stream);
  return e == hipSuccess ? DLS_OK : hip_fail(e, "token_logprobs launch");
}

size_t dls_distill_workspace_size(int64_t rows, int32_t V) {
  return size_ok(rows, V) ? dls::distill_workspace_bytes(rows, V) : 0;
}

dls_status dls_distill_loss(const void* logits, dls_dtype dtype_in, int64_t rows, int32_t V, int64_t row_stride,
                            dls_teacher teacher, const float* grad_loss, float* out_loss, float* out_lse, void* out_grad,
                            int64_t grad_stride, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  const int dtype = enum_bits(dtype_in);
  dls_status s;
  if (!valid_dtype(dtype)) return fail(DLS_ERR_DTYPE, "unknown dtype %d", dtype);
  if ((s = check_rows(rows, V)) != DLS_OK || (s = check_stride(row_stride, V, "row_stride")) != DLS_OK) return s;
  if (out_grad && (s = check_stride(grad_stride, V, "grad_stride")) != DLS_OK) return s;
  if ((s = check_teacher(teacher)) != DLS_OK) return s;
  if (rows == 0) return DLS_OK;
  if (!logits) return fail(DLS_ERR_ARG, "logits is NULL");
  if (!out_loss && !out_lse && !out_grad) return fail(DLS_ERR_ARG, "no output is wanted");
  if ((s = check_teacher_pointers(teacher)) != DLS_OK) return s;
  if (!aligned(logits, elem(dtype)) || !aligned(out_grad, elem(dtype)) || !aligned(out_loss, 4) || !aligned(out_lse, 4) ||
      !aligned(grad_loss, 4))
    return fail(DLS_ERR_ARG, "misaligned pointer");
  if (out_grad == logits && grad_stride != row_stride)
    return fail(DLS_ERR_ARG, "a gradient in place of the logits needs their row stride");
  if ((s = check_workspace(workspace, ws_bytes, dls_distill_workspace_size(rows, V))) != DLS_OK) return s;
  if ((s = check_device()) != DLS_OK) return s;
  dls::DistillArgs a = {};
  a.logits = logits;
  a.dtype = static_cast<dls_dtype>(dtype);
  a.rows = rows;
  a.V = V;
  a.stride = row_stride;
  a.teacher = teacher_args(teacher);
  a.weight = grad_loss;
  a.out_loss = out_loss;
  a.out_lse = out_lse;
  a.grad = out_grad;
  a.grad_stride = grad_stride;
  a.ws = (char*)workspace;
  const hipError_t e = dls::launch_distill_loss(a, (hipStream_t)stream);
  return e == hipSuccess ? DLS_OK : hip_fail(e, "distill_loss launch");
}

dls_status dls_distill_grad(const void* logits, dls_dtype dtype_in, int64_t rows, int32_t V, int64_t row_stride,
                            const float* lse, dls_teacher teacher, const float* grad_loss, void* out_grad,
                            int64_t grad_stride, void* stream) {
  clear_error();
  const int dtype = enum_bits(dtype_in);
  dls_status s;
  if (!valid_dtype(dtype)) return fail(DLS_ERR_DTYPE, "unknown dtype %d", dtype);
  if ((s = check_rows(rows, V)) != DLS_OK || (s = check_stride(row_stride, V, "row_stride")) != DLS_OK ||
      (s = check_stride(grad_stride, V, "grad_stride")) != DLS_OK || (s = check_teacher(teacher)) != DLS_OK)
    return s;
  if (rows == 0) return DLS_OK;
  if (!logits || !lse || !out_grad) return fail(DLS_ERR_ARG, "required pointer is NULL");
  if ((s = check_teacher_pointers(teacher)) != DLS_OK) return s;
  if (!aligned(logits, elem(dtype)) || !aligned(out_grad, elem(dtype)) || !aligned(lse, 4) || !aligned(grad_loss, 4))
    return fail(DLS_ERR_ARG, "misaligned pointer");
  if (out_grad == logits && grad_stride != row_stride)
    return fail(DLS_ERR_ARG, "a gradient in place of the logits needs their row stride");
  if ((s = check_device()) != DLS_OK) return s;
  dls::DistillArgs a = {};
  a.logits = logits;
  a.dtype = static_cast<dls_dtype>(dtype);
  a.rows = rows;
  a.V = V;
  a.stride = row_stride;
  a.teacher = teacher_args(teacher);
  a.weight = grad_loss;
  a.lse = lse;
  a.grad = out_grad;
  a.grad_stride = grad_stride;
  const hipError_t e = dls::launch_distill_grad(a, (hipStream_t)stream);
  return e == hipSuccess ? DLS_OK : hip_fail(e, "distill_grad launch");
}

size_t dls_head_distill_workspace_size(int64_t rows, int32_t V, int32_t r, int32_t k, int with_gradients) {
  if (!size_ok(rows, V) || check_head_sizes(V, r) != DLS_OK || k < 1 || k > kMostK) return 0;
  return dls::head_layout(rows, V, r, k, with_gradients != 0).total;
}

dls_status dls_head_distill(const void* rho, const void* w_vocab, int64_t rows, int32_t V, int32_t r, dls_teacher teacher,
                            const float* grad_loss, float* out_loss, float* out_lse, void* out_d_rho, void* out_d_w,
                            void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  dls_status s;
  if ((s = check_rows(rows, V)) != DLS_OK || (s = check_head_sizes(V, r)) != DLS_OK || (s = check_teacher(teacher)) != DLS_OK)
    return s;
  const bool grads = out_d_rho || out_d_w;
  if (rows == 0 && !out_d_w) return DLS_OK;   // (without rows d_w is 0, and d_rho may be NULL)
  if (rows > 0 && grads && !(out_d_rho && out_d_w)) return fail(DLS_ERR_ARG, "out_d_rho and out_d_w are wanted together");
  if (!w_vocab || (rows > 0 && !rho)) return fail(DLS_ERR_ARG, "required pointer is NULL");
  if (!out_loss && !out_lse && !grads) return fail(DLS_ERR_ARG, "no output is wanted");
  if (rows > 0 && (s = check_teacher_pointers(teacher)) != DLS_OK) return s;
  if (!aligned(rho, 16) || !aligned(w_vocab, 16) || !aligned(out_d_rho, 16) || !aligned(out_d_w, 16) ||
      !aligned(out_loss, 4) || !aligned(out_lse, 4) || !aligned(grad_loss, 4))
    return fail(DLS_ERR_ARG, "misaligned pointer");
  const size_t need = dls_head_distill_workspace_size(rows, V, r, teacher.k, grads);
  if (ws_bytes < need) return fail(DLS_ERR_WORKSPACE, "workspace %zu bytes < %zu required", ws_bytes, need);
  if (need && (!workspace || !aligned(workspace, 256))) return fail(DLS_ERR_ARG, "workspace is NULL or not 256-byte aligned");
  if ((s = check_device()) != DLS_OK) return s;
  dls::HeadDistillArgs a;
  a.rho = rho;
  a.w = w_vocab;
  a.rows = rows;
  a.V = V;
  a.r = r;
  a.teacher = teacher_args(teacher);
  a.weight = grad_loss;
  a.out_loss = out_loss;
  a.out_lse = out_lse;
  a.d_rho = out_d_rho;
  a.d_w = out_d_w;
  a.ws = (char*)workspace;
  const hipError_t e = dls::launch_head_distill(a, (hipStream_t)stream);
  return e == hipSuccess ? DLS_OK : hip_fail(e, "head_distill launch");
}

}  // extern "C"
