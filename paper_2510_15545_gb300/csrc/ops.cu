// ops.cu -- the extern "C" entry points of the operators around a verification
// step: argument checks (before anything touches the GPU) and launches.
#include <algorithm>
#include <array>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <utility>

#include "tt_ops.h"

namespace {

using namespace tt;

// (log2(e) / T and what it scales stay within fp32)
bool temp_ok(float t) { return t >= 1e-36f && t <= 1e36f; }
constexpr double kTwoPi = 6.283185307179586476925;
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

bool rope_plan_ok(const tt_rope_plan& p, int head_dim) {
  return p.turns && (reinterpret_cast<uintptr_t>(p.turns) & 7) == 0 && p.rot_dim >= 2 &&
         p.rot_dim <= head_dim && p.rot_dim % 2 == 0 && (p.interleaved == 0 || p.interleaved == 1) &&
         std::isfinite(p.mscale);
}

// Heads that are written: none shares memory with another.
bool heads_apart(const tt_heads& h, int64_t tokens, int64_t heads, int D) {
  if (!heads_ok(h)) return false;
  if (heads == 1) return tokens == 1 || h.token_stride >= D;
  if (tokens == 1) return h.head_stride >= D;
  const int64_t in = std::min(h.token_stride, h.head_stride);
  const int64_t out = std::max(h.token_stride, h.head_stride);
  // (equal strides would put head h of token i on head h + 1 of token i - 1)
  const int64_t inner = h.token_stride < h.head_stride ? tokens : heads;
  return in >= D && (out - D) / in >= inner - 1 && in != out;
}

// Whether an output is its input, or lies in memory of its own as far as its pointer
// and strides tell.
bool out_ok(const tt_heads& in, const tt_heads& out) {
  return in.data != out.data ||
         (in.token_stride == out.token_stride && in.head_stride == out.head_stride);
}

bool scales_ok(const tt_scales& s) {
  return s.data && s.page_stride >= 0 && s.group_stride >= 0 && s.head_stride >= 0;
}
// Pages of e4m3 elements.
bool pages8_ok(const tt_pages& p, const tt_scales& s) {
  return pages_ok(p) && p.page_stride % 16 == 0 && p.slot_stride % 16 == 0 &&
         p.head_stride % 16 == 0 && scales_ok(s);
}

// Whether runs of `one` elements, at every sum of multiples of three strides (>= 0) up to
// their counts, share no memory, as those of nested dimensions do.
bool entries_apart(int64_t one, std::array<std::pair<int64_t, int64_t>, 3> stride_count) {
  std::sort(stride_count.begin(), stride_count.end());
  int64_t extent = one;  // of what the strides so far reach
  for (const auto& [stride, count] : stride_count) {
    if (count < 2) continue;
    if (stride < extent) return false;
    extent = stride > (INT64_MAX - extent) / (count - 1) ? INT64_MAX : extent + stride * (count - 1);
  }
  return true;
}
// Caches that are written, and their scales.
bool pages_apart(const tt_append* p, const tt_pages& c) {
  return entries_apart(p->head_dim, {{{c.page_stride, p->n_pages}, {c.slot_stride, p->page_size},
                                      {c.head_stride, p->n_heads}}});
}
bool scales_apart(const tt_append* p, const tt_scales& c) {
  return entries_apart(1, {{{c.page_stride, p->n_pages}, {c.group_stride, p->page_size / TT_SCALE_SLOTS},
                            {c.head_stride, p->n_heads}}});
}

// What both tree calls check beyond the sizes, but for their caches.
tt_status tree_ok(const tt_tree* tree, const void* out, const int32_t* status) {
  if (tree->dtype != TT_BF16 && tree->dtype != TT_F16) return TT_ERR_INVALID_ARG;
  if (!(tree->scale > 0.f) || !std::isfinite(tree->scale)) return TT_ERR_INVALID_ARG;
  if (tree->B == 0) return TT_OK;
  if (!tree->tree_off || !tree->cache_len || !status) return TT_ERR_INVALID_ARG;
  if (tree->n_nodes > 0 && (!heads_ok(tree->q) || !heads_ok(tree->k) || !heads_ok(tree->v) ||
                            !aligned16(out)))
    return TT_ERR_INVALID_ARG;
  const int64_t pages = (int64_t(tree->max_len) + tree->page_size - 1) / tree->page_size;
  if (tree->max_len > 0 && (tree->n_pages < 1 || tree->n_pages > INT32_MAX || !tree->page_table ||
                            tree->table_stride < pages))
    return TT_ERR_INVALID_ARG;
  return TT_OK;
}

bool workspace_ok(const void* workspace, size_t bytes, size_t need) {
  return need == 0 || (workspace && bytes >= need &&
                       (reinterpret_cast<uintptr_t>(workspace) & 255) == 0);
}

RopeTensor rope_tensor(const tt_heads& h) {
  return {static_cast<char*>(const_cast<void*>(h.data)), h.token_stride, h.head_stride};
}

// Whether n numbers at a and m at b (NULL: none) share memory.
bool meet(const int32_t* a, int64_t n, const int32_t* b, int64_t m) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return b && x < y + uintptr_t(m) * 4 && y < x + uintptr_t(n) * 4;
}

AppendCache append_cache(const tt_pages& p, const tt_scales& s) {
  return {static_cast<char*>(const_cast<void*>(p.data)), p.page_stride, p.slot_stride,
          p.head_stride, s.data, s.page_stride, s.group_stride, s.head_stride};
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
  const tt_status st = tree_ok(tree, out, status);
  if (st != TT_OK || tree->B == 0) return st;
  if (tree->max_len > 0 && (!pages_ok(tree->k_cache) || !pages_ok(tree->v_cache)))
    return TT_ERR_INVALID_ARG;
  TreeArgs a = tree_args(tree);
  if (!workspace_ok(workspace, workspace_bytes, tree_workspace_bytes(a, device_sms())))
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

size_t tt_tree8_workspace_bytes(const tt_tree* tree) {
  return tree_sizes_ok(tree) ? tree8_workspace_bytes(tree_args(tree), device_sms()) : 0;
}

tt_status tt_tree_attn8(const tt_tree* tree, const tt_scales* k_scale, const tt_scales* v_scale,
                        void* workspace, size_t workspace_bytes, void* out, float* lse,
                        int32_t* status, void* stream) {
  if (!tree_sizes_ok(tree) || !k_scale || !v_scale) return TT_ERR_INVALID_ARG;
  const tt_status st = tree_ok(tree, out, status);
  if (st != TT_OK || tree->B == 0) return st;
  if (tree->max_len > 0 &&
      (!pages8_ok(tree->k_cache, *k_scale) || !pages8_ok(tree->v_cache, *v_scale)))
    return TT_ERR_INVALID_ARG;
  TreeArgs a = tree_args(tree);
  if (!workspace_ok(workspace, workspace_bytes, tree8_workspace_bytes(a, device_sms())))
    return TT_ERR_INVALID_ARG;
  if (!tree8_fits(a, device_sms())) return TT_ERR_UNSUPPORTED;
  a.ws = static_cast<char*>(workspace);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.status = status;
  const TreeScales sc = {
      {k_scale->data, k_scale->page_stride, k_scale->group_stride, k_scale->head_stride},
      {v_scale->data, v_scale->page_stride, v_scale->group_stride, v_scale->head_stride}};
  cudaError_t e = load_kernels();
  if (e == cudaSuccess)
    e = launch_tree8(a, sc, tree->dtype, static_cast<cudaStream_t>(stream), device_sms());
  return e == cudaSuccess ? TT_OK : record_cuda_error(e);
}

tt_status tt_rope_freqs(const tt_rope_config* c, double* freqs) {
  if (!c || !freqs || c->rot_dim < 2 || c->rot_dim > 256 || c->rot_dim % 2 != 0)
    return TT_ERR_INVALID_ARG;
  if (!(c->base > 0.0) || !std::isfinite(c->base)) return TT_ERR_INVALID_ARG;
  if (c->scaling < TT_ROPE_PLAIN || c->scaling > TT_ROPE_PARTS) return TT_ERR_INVALID_ARG;
  if (c->scaling != TT_ROPE_PLAIN && (!(c->factor > 0.0) || !std::isfinite(c->factor)))
    return TT_ERR_INVALID_ARG;
  if (c->scaling == TT_ROPE_BASE && c->rot_dim < 4) return TT_ERR_INVALID_ARG;
  if (c->scaling == TT_ROPE_PARTS &&
      (!(c->original > 0.0) || !std::isfinite(c->original) || !std::isfinite(c->low) ||
       !std::isfinite(c->high) || !(c->low < c->high)))
    return TT_ERR_INVALID_ARG;
  const double d = c->rot_dim;
  const double base =
      c->scaling == TT_ROPE_BASE ? c->base * std::pow(c->factor, d / (d - 2.0)) : c->base;
  for (int i = 0; i < c->rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / d);
    if (c->scaling == TT_ROPE_LINEAR) f /= c->factor;
    if (c->scaling == TT_ROPE_PARTS) {
      const double r = c->original * f / kTwoPi;
      const double g = std::min(1.0, std::max(0.0, (r - c->low) / (c->high - c->low)));
      f *= (1.0 - g) / c->factor + g;
    }
    freqs[i] = f;
  }
  return TT_OK;
}

tt_status tt_rope_turns(const double* freqs, int32_t n, uint64_t* turns) {
  if (n < 0 || (n > 0 && (!freqs || !turns))) return TT_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i)
    if (!std::isfinite(freqs[i])) return TT_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const double t = freqs[i] / kTwoPi, part = t - std::floor(t);
    // (a tiny negative angle's part may round to a whole turn: none)
    turns[i] = part < 1.0 ? uint64_t(std::ldexp(part, 64)) : 0;
  }
  return TT_OK;
}

tt_status tt_rope(const tt_rotate* r, void* stream) {
  if (!r || r->n_tokens < 0 || r->dtype < TT_F32 || r->dtype > TT_F16 || r->head_dim < 8 ||
      r->head_dim > 256 || r->head_dim % 8 != 0 || r->n_q_heads < 1 || r->n_k_heads < 0 ||
      (r->transpose != 0 && r->transpose != 1))
    return TT_ERR_INVALID_ARG;
  if (!rope_plan_ok(r->plan, r->head_dim)) return TT_ERR_INVALID_ARG;
  if (r->n_tokens == 0) return TT_OK;
  if (!r->positions || !heads_ok(r->q) || !out_ok(r->q, r->q_out) ||
      !heads_apart(r->q_out, r->n_tokens, r->n_q_heads, r->head_dim))
    return TT_ERR_INVALID_ARG;
  if (r->n_k_heads > 0 && (!heads_ok(r->k) || !out_ok(r->k, r->k_out) ||
                           !heads_apart(r->k_out, r->n_tokens, r->n_k_heads, r->head_dim)))
    return TT_ERR_INVALID_ARG;
  if (int64_t(r->n_q_heads) + r->n_k_heads > 65535) return TT_ERR_UNSUPPORTED;
  RopeArgs a;
  std::memset(&a, 0, sizeof a);
  a.n_tokens = r->n_tokens;
  a.D = r->head_dim;
  a.Hq = r->n_q_heads;
  a.Hk = r->n_k_heads;
  a.rot_dim = r->plan.rot_dim;
  a.interleaved = r->plan.interleaved;
  a.back = r->transpose;
  a.mscale = r->plan.mscale;
  a.positions = r->positions;
  a.turns = r->plan.turns;
  a.q = rope_tensor(r->q);
  a.k = rope_tensor(r->k);
  a.q_out = rope_tensor(r->q_out);
  a.k_out = rope_tensor(r->k_out);
  cudaError_t e = load_kernels();
  if (e == cudaSuccess)
    e = launch_rope(a, r->dtype, static_cast<cudaStream_t>(stream), device_sms());
  return e == cudaSuccess ? TT_OK : record_cuda_error(e);
}

tt_status tt_cache_append(const tt_append* p, const tt_rope_plan* rope, int32_t* new_len,
                          int32_t* status, void* stream) {
  if (!p || p->B < 0 || p->n_tokens < 0 || p->max_new < 1 ||
      (p->dtype != TT_BF16 && p->dtype != TT_F16) ||
      (p->cache_dtype != p->dtype && p->cache_dtype != TT_E4M3) || p->n_heads < 1 ||
      (p->head_dim != 64 && p->head_dim != 128) || p->page_size < 16 || p->page_size % 16 != 0 ||
      p->page_size > 1 << 20 || p->max_len < 0 || p->max_len > 1 << 30)
    return TT_ERR_INVALID_ARG;
  if (rope && !rope_plan_ok(*rope, p->head_dim)) return TT_ERR_INVALID_ARG;
  if (p->B == 0) return TT_OK;
  if (!p->token_off || !p->cache_len || !status) return TT_ERR_INVALID_ARG;
  // (what some CTAs write, others still read)
  const int64_t B = p->B;
  for (const int32_t* out : {static_cast<const int32_t*>(new_len), static_cast<const int32_t*>(status)})
    if (out && (meet(out, B, p->cache_len, B) || meet(out, B, p->token_off, B + 1) ||
                meet(out, B, p->keep, B) || meet(out, B, p->path, p->n_tokens)))
      return TT_ERR_INVALID_ARG;
  if (new_len && meet(new_len, B, status, B)) return TT_ERR_INVALID_ARG;
  if (p->n_tokens > 0 && (!heads_ok(p->k) || !heads_ok(p->v))) return TT_ERR_INVALID_ARG;
  const bool held8 = p->cache_dtype == TT_E4M3;
  const int64_t pages = (int64_t(p->max_len) + p->page_size - 1) / p->page_size;
  if (p->max_len > 0) {
    if (held8 ? !pages8_ok(p->k_cache, p->k_scale) || !pages8_ok(p->v_cache, p->v_scale)
              : !pages_ok(p->k_cache) || !pages_ok(p->v_cache))
      return TT_ERR_INVALID_ARG;
    if (p->k_cache.data == p->v_cache.data || (held8 && p->k_scale.data == p->v_scale.data))
      return TT_ERR_INVALID_ARG;
    if (p->n_pages < 1 || p->n_pages > INT32_MAX || !p->page_table || p->table_stride < pages)
      return TT_ERR_INVALID_ARG;
    if (!pages_apart(p, p->k_cache) || !pages_apart(p, p->v_cache) ||
        (held8 && (!scales_apart(p, p->k_scale) || !scales_apart(p, p->v_scale))))
      return TT_ERR_INVALID_ARG;
  }
  // (a CTA's threads share the requests out by numbers of 32 bits)
  if (p->B > 1 << 30) return TT_ERR_UNSUPPORTED;
  AppendArgs a;
  std::memset(&a, 0, sizeof a);
  a.B = p->B;
  a.n_tokens = p->n_tokens;
  a.max_new = p->max_new;
  a.H = p->n_heads;
  a.D = p->head_dim;
  a.page_size = p->page_size;
  a.max_len = p->max_len;
  a.token_off = p->token_off;
  a.keep = p->keep;
  a.path = p->path;
  a.positions = p->positions;
  a.cache_len = p->cache_len;
  a.page_table = p->page_table;
  a.n_pages = p->n_pages;
  a.table_stride = p->table_stride;
  a.k = rope_tensor(p->k);
  a.v = rope_tensor(p->v);
  a.k_cache = append_cache(p->k_cache, p->k_scale);
  a.v_cache = append_cache(p->v_cache, p->v_scale);
  if (rope) {
    a.rot_dim = rope->rot_dim;
    a.interleaved = rope->interleaved;
    a.mscale = rope->mscale;
    a.turns = rope->turns;
  }
  a.new_len = new_len;
  a.status = status;
  cudaError_t e = load_kernels();
  if (e == cudaSuccess)
    e = launch_append(a, p->dtype, held8, static_cast<cudaStream_t>(stream), device_sms());
  return e == cudaSuccess ? TT_OK : record_cuda_error(e);
}

}  // extern "C"
