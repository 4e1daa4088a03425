// ops.cu -- the extern "C" entry points of the operators around a verification
// step: argument checks (before anything touches the GPU) and launches.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "tt_ops.h"

namespace {

using namespace tt;

// (log2(e) / T and what it scales stay within fp32)
bool temp_ok(float t) { return t >= 1e-36f && t <= 1e36f; }
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

bool aligned16(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0; }
bool heads_ok(const tt_heads& h) {
  return aligned16(h.data) && stride_ok(h.token_stride) && stride_ok(h.head_stride);
}
bool pages_ok(const tt_pages& p) {
  return aligned16(p.data) && stride_ok(p.page_stride) && stride_ok(p.slot_stride) &&
         stride_ok(p.head_stride);
}

// The sizes of a tree call, on which its workspace depends.
bool tree_sizes_ok(const tt_tree* t) {
  if (!t || t->B < 0 || t->n_nodes < 0 || t->max_nodes < 1 || t->max_nodes > TT_MAX_TREE)
    return false;
  if (t->n_kv_heads < 1 || t->n_q_heads < 1 || t->n_q_heads % t->n_kv_heads != 0 ||
      t->n_q_heads / t->n_kv_heads > 128)
    return false;
  return (t->head_dim == 64 || t->head_dim == 128) && t->page_size >= 16 &&
         t->page_size % 16 == 0 && t->page_size <= 1 << 20 && t->max_len >= 0 &&
         t->max_len <= 1 << 30;
}

TreeArgs tree_args(const tt_tree* t) {
  TreeArgs a;
  std::memset(&a, 0, sizeof a);
  a.B = t->B;
  a.n_nodes = t->n_nodes;
  a.max_nodes = t->max_nodes;
  a.Hq = t->n_q_heads;
  a.Hkv = t->n_kv_heads;
  a.D = t->head_dim;
  a.tree_off = t->tree_off;
  a.parents = t->parents;
  a.q = static_cast<const char*>(t->q.data);
  a.q_token = t->q.token_stride;
  a.q_head = t->q.head_stride;
  a.k = static_cast<const char*>(t->k.data);
  a.k_token = t->k.token_stride;
  a.k_head = t->k.head_stride;
  a.v = static_cast<const char*>(t->v.data);
  a.v_token = t->v.token_stride;
  a.v_head = t->v.head_stride;
  a.kc = static_cast<const char*>(t->k_cache.data);
  a.kc_page = t->k_cache.page_stride;
  a.kc_slot = t->k_cache.slot_stride;
  a.kc_head = t->k_cache.head_stride;
  a.vc = static_cast<const char*>(t->v_cache.data);
  a.vc_page = t->v_cache.page_stride;
  a.vc_slot = t->v_cache.slot_stride;
  a.vc_head = t->v_cache.head_stride;
  a.n_pages = t->n_pages;
  a.page_size = t->page_size;
  a.page_table = t->page_table;
  a.table_stride = t->table_stride;
  a.cache_len = t->cache_len;
  a.max_len = t->max_len;
  a.scale = t->scale;
  return a;
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
  if (e == cudaSuccess)
    e = launch_distill(a, student->dtype, static_cast<cudaStream_t>(stream), device_sms());
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

size_t tt_tree_workspace_bytes(const tt_tree* tree) {
  return tree_sizes_ok(tree) ? tree_workspace_bytes(tree_args(tree), device_sms()) : 0;
}

tt_status tt_tree_attn(const tt_tree* tree, void* workspace, size_t workspace_bytes, void* out,
                       float* lse, int32_t* status, void* stream) {
  if (!tree_sizes_ok(tree)) return TT_ERR_INVALID_ARG;
  if (tree->dtype != TT_BF16 && tree->dtype != TT_F16) return TT_ERR_INVALID_ARG;
  if (!(tree->scale > 0.f) || !std::isfinite(tree->scale)) return TT_ERR_INVALID_ARG;
  if (tree->B == 0) return TT_OK;
  if (!tree->tree_off || !tree->cache_len || !status) return TT_ERR_INVALID_ARG;
  if (tree->n_nodes > 0 && (!heads_ok(tree->q) || !heads_ok(tree->k) || !heads_ok(tree->v) ||
                            !aligned16(out)))
    return TT_ERR_INVALID_ARG;
  const int64_t pages = (int64_t(tree->max_len) + tree->page_size - 1) / tree->page_size;
  if (tree->max_len > 0 &&
      (!pages_ok(tree->k_cache) || !pages_ok(tree->v_cache) || tree->n_pages < 1 ||
       tree->n_pages > INT32_MAX || !tree->page_table || tree->table_stride < pages))
    return TT_ERR_INVALID_ARG;
  TreeArgs a = tree_args(tree);
  const size_t need = tree_workspace_bytes(a, device_sms());
  if (need > 0 && (!workspace || workspace_bytes < need ||
                   (reinterpret_cast<uintptr_t>(workspace) & 255) != 0))
    return TT_ERR_INVALID_ARG;
  if (!tree_fits(a, device_sms())) return TT_ERR_UNSUPPORTED;
  a.ws = static_cast<char*>(workspace);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.status = status;
  cudaError_t e = load_kernels();
  if (e == cudaSuccess)
    e = launch_tree(a, tree->dtype, static_cast<cudaStream_t>(stream), device_sms());
  return e == cudaSuccess ? TT_OK : record_cuda_error(e);
}

}  // extern "C"
