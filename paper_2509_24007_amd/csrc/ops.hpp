// Operators on tensors that the caller names (not those of a context): declarations shared by their kernels and entry points.
#pragma once
#include "internal.hpp"

namespace sdlm {

// ---- drawing tokens from logits (sample.hip)
constexpr int SAMPLE_MAX_V = 1 << 19;   // weights are 44-bit fixed point: their sum over a row stays inside 64 bits
constexpr int SAMPLE_MAX_ROWS = 1 << 20;
bool sample_fits(int rows, int vocab);   // one launch holds them
size_t sample_workspace_bytes(int rows, int vocab);
void launch_sample(hipStream_t s, const sdlm_sample_args &a, void *workspace);

// ---- attention of token trees over the cache (tree_attn.hip)
constexpr int TREE_MAX_NODES = 1024;
bool tree_fits(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes);   // the launch's counters hold them
size_t tree_workspace_bytes(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes, int max_len);
size_t tree_workspace_least(int n_kv_heads, int head_dim, int dtype);   // what launch_tree_attention needs at least, whatever the sizes of the call are
void launch_tree_attention(hipStream_t s, const sdlm_kv &kv, int layer, const sdlm_tree_args &t, void *workspace, size_t workspace_bytes);

// ---- pages (kv_pages.hip)
size_t fork_workspace_bytes(const sdlm_kv &kv);
void launch_fork(hipStream_t s, const sdlm_kv &kv, const int32_t *parent, int n_new, int share, int32_t *status, void *workspace);
void launch_compact(hipStream_t s, const sdlm_kv &kv, const int32_t *start, const int32_t *node_table, int node_pages, const int32_t *node_base, const int32_t *path,
                    int path_stride, const int32_t *path_len, int n_seqs, int max_path);

}  // namespace sdlm
