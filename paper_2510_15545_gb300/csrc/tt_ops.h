// tt_ops.h -- arguments and launchers of the operators around a verification
// step: log probabilities of logits rows (logprob.cu), a student's loss against a
// teacher's top log probabilities (distill.cu), attention of drafted tokens over a
// paged cache (tree.cu; in 8 bits, tree8.cu and tree8_few.cu), rotary positions
// (rope.cu), appending to paged caches (append.cu).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "tt.h"

namespace tt {

// What the entry points share (api.cu): every kernel loaded on the current
// device, its SM count, logits rows that the kernels take, a failed call's code.
cudaError_t load_kernels();
int device_sms();
bool rows_usable(const tt_logits* L, int64_t rows);
tt_status record_cuda_error(cudaError_t e);
// Test hook of the bounded waits (rowpass.cu, whose launches and those of the
// operators that wait for copies are counted together): the CTA whose copies are
// withheld and the wait limit of the next launch; false (and the defaults) when off.
bool next_launch_stall(int32_t* cta, uint64_t* wait_ns);

struct LogprobArgs {
  const char* data;
  int64_t stride_bytes;
  int64_t rows;
  int V;
  float temp, scale;  // T, log2(e) / T
  int top_n;
  const int32_t* ids;
  tt_logprobs_out out;
  int split, share;  // CTAs per row and columns of each, and
  float reach;       // 300 in the units of z (filled in by the launcher)
};

cudaError_t launch_logprobs(const LogprobArgs& args, int dt, cudaStream_t stream, int sm_count);
cudaError_t preload_logprobs();

struct DistillArgs {
  const char* data;  // student logits
  int64_t stride_bytes;
  int64_t rows;
  int V, K, tail;
  float temp, scale;  // T, log2(e) / T
  const int32_t* ids;   // [rows * K]
  const float* logp;    // [rows * K]
  const float* weight;  // [rows] or NULL
  float* loss;
  float* stats;  // [rows * 4]: max z and sum of 2^((z - max) scale), of all columns and of
                 // those outside the list
  int32_t* status;
  char* grad;  // NULL: the forward call alone
  int64_t grad_stride_bytes;
  // filled in by the launcher:
  int split, share;  // CTAs per row and columns of each
  int stall;         // the CTA whose copies a test withholds, or -1
  uint64_t wait_ns;  // limit of a wait
};

int distill_max_cols(int dt);
cudaError_t launch_distill(const DistillArgs& args, int dt, cudaStream_t stream, int sm_count);
cudaError_t launch_distill_grad(const DistillArgs& args, int dt, cudaStream_t stream);
cudaError_t preload_distill();

struct TreeArgs {
  int B, n_nodes, max_nodes, Hq, Hkv, D;
  const int32_t* tree_off;
  const int32_t* parents;  // NULL: chains
  const char *q, *k, *v;   // strides below in elements
  int64_t q_token, q_head, k_token, k_head, v_token, v_head;
  const char *kc, *vc;
  int64_t kc_page, kc_slot, kc_head, vc_page, vc_slot, vc_head;
  int64_t n_pages;
  int page_size;
  const int32_t* page_table;
  int64_t table_stride;
  const int32_t* cache_len;
  int max_len;
  float scale;
  char* ws;
  char* out;
  float* lse;
  int32_t* status;
};

size_t tree_workspace_bytes(const TreeArgs& args, int sm_count);
bool tree_fits(const TreeArgs& args, int sm_count);
cudaError_t launch_tree(const TreeArgs& args, int dt, cudaStream_t stream, int sm_count);
cudaError_t preload_tree();

struct RopeTensor {
  char* data;  // strides in elements
  int64_t token, head;
};
struct RopeArgs {
  int n_tokens, D, Hq, Hk, rot_dim, interleaved, back;
  float mscale;
  const int32_t* positions;
  const uint64_t* turns;
  RopeTensor q, k, q_out, k_out;
};

cudaError_t launch_rope(const RopeArgs& args, int dt, cudaStream_t stream, int sm_count);
cudaError_t preload_rope();

struct AppendCache {
  char* data;  // strides in elements
  int64_t page, slot, head;
  uint8_t* scale;  // strides in bytes
  int64_t scale_page, scale_group, scale_head;
};
struct AppendArgs {
  int B, n_tokens, max_new, H, D, page_size, max_len;
  const int32_t *token_off, *keep, *path, *positions, *cache_len, *page_table;
  int64_t n_pages, table_stride;
  RopeTensor k, v;
  AppendCache k_cache, v_cache;
  int rot_dim, interleaved;  // rot_dim 0: no rotation
  float mscale;
  const uint64_t* turns;
  int32_t *new_len, *status;
};

cudaError_t launch_append(const AppendArgs& args, int dt, bool held8, cudaStream_t stream,
                          int sm_count);
cudaError_t preload_append();

struct TreeScale {
  const uint8_t* data;  // strides in bytes
  int64_t page, group, head;
};
struct TreeScales {
  TreeScale k, v;
};

size_t tree8_workspace_bytes(const TreeArgs& args, int sm_count);
bool tree8_fits(const TreeArgs& args, int sm_count);
cudaError_t launch_tree8(const TreeArgs& args, const TreeScales& scales, int dt,
                         cudaStream_t stream, int sm_count);
cudaError_t preload_tree8();

}  // namespace tt
