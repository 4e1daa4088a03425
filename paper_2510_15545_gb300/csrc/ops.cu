// ops.cu -- the extern "C" entry points of the operators around a verification
// step: argument checks (before anything touches the GPU) and launches.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "tt_ops.h"

namespace {

using namespace tt;

bool temp_ok(float t) { return t > 0.f && std::isfinite(t); }
float log2e_over(float t) { return float(1.4426950408889634 / double(t)); }

int elem_size(const tt_logits* L) { return L->dtype == TT_F32 ? 4 : 2; }

// The arguments that both distillation calls take; grad may be NULL.
tt_status distill_args(const tt_logits* student, const tt_teacher* teacher, float temp,
                       int32_t tail, const float* weight, const tt_logits* grad, DistillArgs* a) {
  if (!rows_usable(student, student->n_rows)) return TT_ERR_INVALID_ARG;
  if (teacher->k > 0 && (!teacher->ids || !teacher->logp)) return TT_ERR_INVALID_ARG;
  if (grad && (!rows_usable(grad, student->n_rows) || grad->dtype != student->dtype ||
               grad->n_cols != student->n_cols))
    return TT_ERR_INVALID_ARG;
  if (student->n_rows > INT32_MAX / 1024 || student->n_cols > distill_max_cols(student->dtype))
    return TT_ERR_UNSUPPORTED;
  std::memset(a, 0, sizeof *a);
  a->data = static_cast<const char*>(student->data);
  a->stride_bytes = student->row_stride * elem_size(student);
  a->rows = student->n_rows;
  a->V = student->n_cols;
  a->K = teacher->k;
  a->tail = tail;
  a->temp = temp;
  a->scale = log2e_over(temp);
  a->ids = teacher->ids;
  a->logp = teacher->logp;
  a->weight = weight;
  if (grad) {
    a->grad = static_cast<char*>(const_cast<void*>(grad->data));
    a->grad_stride_bytes = grad->row_stride * elem_size(grad);
  }
  return TT_OK;
}

bool distill_ok(const tt_logits* student, const tt_teacher* teacher, float temp, int32_t tail) {
  return student && student->n_rows >= 0 && teacher && teacher->k >= 0 &&
         teacher->k <= TT_MAX_DISTILL_K && temp_ok(temp) && (tail == 0 || tail == 1);
}

}  // namespace

extern "C" {

tt_status tt_logprobs(const tt_logits* rows, const int32_t* ids, float temp, int32_t top_n,
                      const tt_logprobs_out* out, void* stream) {
  if (!rows || rows->n_rows < 0 || !temp_ok(temp) || !out) return TT_ERR_INVALID_ARG;
  if (top_n < 0 || top_n > TT_MAX_TOP_K) return TT_ERR_INVALID_ARG;
  if (rows->n_rows == 0) return TT_OK;
  if (!rows_usable(rows, rows->n_rows) || !out->status) return TT_ERR_INVALID_ARG;
  if ((out->logprob || out->rank) && !ids) return TT_ERR_INVALID_ARG;
  if (rows->n_rows > INT32_MAX) return TT_ERR_UNSUPPORTED;
  LogprobArgs a;
  std::memset(&a, 0, sizeof a);
  a.data = static_cast<const char*>(rows->data);
  a.stride_bytes = rows->row_stride * elem_size(rows);
  a.rows = rows->n_rows;
  a.V = rows->n_cols;
  a.temp = temp;
  a.scale = log2e_over(temp);
  a.top_n = out->top_ids || out->top_logprobs ? top_n : 0;
  a.ids = ids;
  a.out = *out;
  cudaError_t e = load_kernels();
  if (e == cudaSuccess)
    e = launch_logprobs(a, rows->dtype, static_cast<cudaStream_t>(stream), device_sms());
  return e == cudaSuccess ? TT_OK : record_cuda_error(e);
}

tt_status tt_distill(const tt_logits* student, const tt_teacher* teacher, float temp,
                     int32_t tail, const float* weight, float* loss, float* stats,
                     const tt_logits* grad, int32_t* status, void* stream) {
  if (!distill_ok(student, teacher, temp, tail)) return TT_ERR_INVALID_ARG;
  if (student->n_rows == 0) return TT_OK;
  if (!status || (reinterpret_cast<uintptr_t>(stats) & 15) != 0) return TT_ERR_INVALID_ARG;
  DistillArgs a;
  const tt_status st = distill_args(student, teacher, temp, tail, weight, grad, &a);
  if (st != TT_OK) return st;
  a.loss = loss;
  a.stats = stats;
  a.status = status;
  cudaError_t e = load_kernels();
  if (e == cudaSuccess) e = launch_distill(a, student->dtype, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? TT_OK : record_cuda_error(e);
}

tt_status tt_distill_grad(const tt_logits* student, const tt_teacher* teacher, float temp,
                          int32_t tail, const float* weight, const float* stats,
                          const tt_logits* grad, void* stream) {
  if (!distill_ok(student, teacher, temp, tail)) return TT_ERR_INVALID_ARG;
  if (student->n_rows == 0) return TT_OK;
  if (!grad || !stats || (reinterpret_cast<uintptr_t>(stats) & 15) != 0) return TT_ERR_INVALID_ARG;
  DistillArgs a;
  const tt_status st = distill_args(student, teacher, temp, tail, weight, grad, &a);
  if (st != TT_OK) return st;
  a.stats = const_cast<float*>(stats);
  cudaError_t e = load_kernels();
  if (e == cudaSuccess)
    e = launch_distill_grad(a, student->dtype, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? TT_OK : record_cuda_error(e);
}

}  // extern "C"
