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
  a.stride_bytes = rows->row_stride * (rows->dtype == TT_F32 ? 4 : 2);
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

}  // extern "C"
