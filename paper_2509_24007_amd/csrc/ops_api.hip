// Entry points of the operators on the caller's tensors: checks of everything that the host can see, then the launches.
#include <stdarg.h>
#include <stdio.h>

#include "ops.hpp"

using namespace sdlm;

namespace {

thread_local char g_err[256] = "";

int bad(int code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return code;
}

int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SDLM_OK : bad(SDLM_EHIP, "%s: %s", what, hipGetErrorString(e));
}

constexpr int MAX_TABLE = 1 << 26;   // entries of a sequence's table: positions fit 31 bits
constexpr int MAX_SEQS = 1 << 20, MAX_HEADS = 65535, MAX_LAYER_HEADS = 1 << 23;   // grids: workgroups along y, threads along x

bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int check_workspace(const void *w, size_t have, size_t need)
{
    if (!w || !aligned(w, 256)) return bad(SDLM_EINVAL, "workspace must be a 256-byte aligned device pointer");
    if (have < need) return bad(SDLM_ECAPACITY, "workspace has %zu bytes, %zu needed", have, need);
    return SDLM_OK;
}

// pages: the call hands out pages too
int check_kv(const sdlm_kv *kv, bool pages)
{
    if (!kv) return bad(SDLM_EINVAL, "null cache");
    if (!kv->pool || !aligned(kv->pool, 16)) return bad(SDLM_EINVAL, "pool must be a 16-byte aligned device pointer");
    if (kv->dtype != 0 && kv->dtype != 1) return bad(SDLM_EINVAL, "dtype must be 0 (fp32) or 1 (bf16)");
    if (kv->head_dim != 32 && kv->head_dim != 64 && kv->head_dim != 96 && kv->head_dim != 128) return bad(SDLM_EINVAL, "head_dim must be 32, 64, 96 or 128");
    if (kv->n_layers < 1 || kv->n_tiles < 1 || kv->n_kv_heads < 1 || kv->max_seqs < 1 || kv->pages_per_seq < 1) return bad(SDLM_EINVAL, "bad cache sizes");
    if (kv->pages_per_seq > MAX_TABLE) return bad(SDLM_EINVAL, "pages_per_seq is at most %d", MAX_TABLE);
    if (kv->n_kv_heads > MAX_HEADS || (long)kv->n_layers * kv->n_kv_heads > MAX_LAYER_HEADS) return bad(SDLM_EINVAL, "too many layers and heads: n_kv_heads is at most %d, n_layers * n_kv_heads %d", MAX_HEADS, MAX_LAYER_HEADS);
    if (kv->max_seqs > MAX_SEQS) return bad(SDLM_EINVAL, "max_seqs is at most %d", MAX_SEQS);
    if (kv->layer_stride < (int64_t)(kv->n_layers > 1 ? kv->n_tiles : 0) * kv->n_kv_heads * 2 * PAGE * kv->head_dim || kv->layer_stride % (kv->dtype == 0 ? 4 : 8))
        return bad(SDLM_EINVAL, "layer_stride must hold the tiles of a layer and be a multiple of 16 bytes");
    if (!kv->page_table || !kv->lengths) return bad(SDLM_EINVAL, "page_table and lengths are required");
    if (pages) {
        if (kv->n_pages < 1 || kv->n_pages > kv->n_tiles) return bad(SDLM_EINVAL, "n_pages must be 1 .. n_tiles");
        if (!kv->backed || !kv->page_refs || !kv->free_pages || !kv->free_count) return bad(SDLM_EINVAL, "backed, page_refs, free_pages and free_count are required");
        if ((long)kv->max_seqs * kv->pages_per_seq > (1l << 30)) return bad(SDLM_EINVAL, "the page table is too large");
    }
    return SDLM_OK;
}

bool sample_sizes(int rows, int vocab) { return rows >= 0 && vocab >= 1 && vocab <= SAMPLE_MAX_V && sample_fits(rows, vocab); }

bool tree_sizes(int n_q_heads, int n_kv_heads, int n_seqs, int max_nodes, int max_len)
{
    return n_q_heads >= 1 && n_q_heads <= MAX_HEADS && n_q_heads % n_kv_heads == 0 && n_seqs >= 0 && max_nodes >= 1 && max_nodes <= TREE_MAX_NODES && max_len >= 0;
}

}  // namespace

extern "C" {

const char *sdlm_op_error(void) { return g_err; }

size_t sdlm_sample_workspace_bytes(int32_t rows, int32_t vocab) { return sample_sizes(rows, vocab) ? sample_workspace_bytes(rows, vocab) : 0; }

int sdlm_sample(const sdlm_sample_args *a, void *workspace, size_t bytes, void *hip_stream)
{
    if (!a) return bad(SDLM_EINVAL, "null arguments");
    if (!sample_sizes(a->rows, a->vocab)) return bad(SDLM_EINVAL, "%d rows of %d logits: rows must be 0 .. %d, vocab 1 .. %d, and a launch hold them", a->rows, a->vocab, SAMPLE_MAX_ROWS, SAMPLE_MAX_V);
    if (a->dtype != 0 && a->dtype != 1) return bad(SDLM_EINVAL, "dtype must be 0 (fp32) or 1 (bf16)");
    if (a->row_stride < a->vocab) return bad(SDLM_EINVAL, "row_stride is less than vocab");
    if (a->rows == 0) return SDLM_OK;
    if (!a->logits || !a->u || !a->ids) return bad(SDLM_EINVAL, "logits, u and ids are required");
    if (!aligned(a->logits, a->dtype == 0 ? 4 : 2)) return bad(SDLM_EINVAL, "logits must be aligned to their element");
    const int rc = check_workspace(workspace, bytes, sample_workspace_bytes(a->rows, a->vocab));
    if (rc) return rc;
    launch_sample((hipStream_t)hip_stream, *a, workspace);
    return launched("sdlm_sample");
}

size_t sdlm_tree_attention_workspace_bytes(const sdlm_kv *kv, int32_t n_q_heads, int32_t n_seqs, int32_t max_nodes, int32_t max_len)
{
    if (check_kv(kv, false)) return 0;
    if (!tree_sizes(n_q_heads, kv->n_kv_heads, n_seqs, max_nodes, max_len)) {
        bad(SDLM_EINVAL, "n_q_heads must be a multiple of n_kv_heads up to %d, max_nodes 1 .. %d, n_seqs and max_len not negative", MAX_HEADS, TREE_MAX_NODES);
        return 0;
    }
    if (!tree_fits(*kv, n_q_heads, n_seqs, max_nodes)) {
        bad(SDLM_EINVAL, "%d sequences of %d pages with %d nodes each are too many for one launch", n_seqs, kv->pages_per_seq, max_nodes);
        return 0;
    }
    return tree_workspace_bytes(*kv, n_q_heads, n_seqs, max_nodes, max_len);
}

int sdlm_tree_attention(const sdlm_kv *kv, int32_t layer, const sdlm_tree_args *t, void *workspace, size_t bytes, void *hip_stream)
{
    int rc = check_kv(kv, false);
    if (rc) return rc;
    if (!t) return bad(SDLM_EINVAL, "null arguments");
    if (layer < 0 || layer >= kv->n_layers) return bad(SDLM_EINVAL, "layer %d outside 0..%d", layer, kv->n_layers - 1);
    if (!tree_sizes(t->n_q_heads, kv->n_kv_heads, t->n_seqs, t->max_nodes, t->max_len))
        return bad(SDLM_EINVAL, "n_q_heads must be a multiple of n_kv_heads up to %d, max_nodes 1 .. %d, n_seqs and max_len not negative", MAX_HEADS, TREE_MAX_NODES);
    if (t->n_seqs > kv->max_seqs) return bad(SDLM_EINVAL, "%d sequences, the cache has %d", t->n_seqs, kv->max_seqs);
    if (t->n_rows < 0 || (long)t->n_rows > (long)t->n_seqs * t->max_nodes) return bad(SDLM_EINVAL, "%d rows for %d sequences of at most %d nodes", t->n_rows, t->n_seqs, t->max_nodes);
    if (t->mask_words < (t->max_nodes + 63) / 64) return bad(SDLM_EINVAL, "mask_words is too small for max_nodes");
    if (t->node_pages < 1 || t->node_pages > MAX_TABLE) return bad(SDLM_EINVAL, "node_pages must be 1 .. %d", MAX_TABLE);
    const int64_t row = (int64_t)t->n_q_heads * kv->head_dim, vec = kv->dtype == 0 ? 4 : 8;
    if (t->q_stride < row || t->out_stride < row || t->q_stride % vec || t->out_stride % vec) return bad(SDLM_EINVAL, "q_stride and out_stride must hold a row and be multiples of 16 bytes");
    if (!tree_fits(*kv, t->n_q_heads, t->n_seqs, t->max_nodes)) return bad(SDLM_EINVAL, "%d sequences of %d pages with %d nodes each are too many for one launch", t->n_seqs, kv->pages_per_seq, t->max_nodes);
    if (t->n_rows == 0 || t->n_seqs == 0) return SDLM_OK;
    if (!t->q || !t->out || !t->node_offsets || !t->mask || !t->node_table) return bad(SDLM_EINVAL, "q, out, node_offsets, mask and node_table are required");
    if (!aligned(t->q, 16) || !aligned(t->out, 16)) return bad(SDLM_EINVAL, "q and out must be 16-byte aligned");
    if ((rc = check_workspace(workspace, bytes, tree_workspace_bytes(*kv, t->n_q_heads, t->n_seqs, t->max_nodes, t->max_len)))) return rc;
    launch_tree_attention((hipStream_t)hip_stream, *kv, layer, *t, workspace, bytes);
    return launched("sdlm_tree_attention");
}

size_t sdlm_kv_fork_workspace_bytes(const sdlm_kv *kv) { return check_kv(kv, true) ? 0 : fork_workspace_bytes(*kv); }

int sdlm_kv_fork(const sdlm_kv *kv, const int32_t *parent, int32_t n_new, int32_t share, int32_t *status, void *workspace, size_t bytes, void *hip_stream)
{
    int rc = check_kv(kv, true);
    if (rc) return rc;
    if (n_new < 0 || n_new > kv->max_seqs) return bad(SDLM_EINVAL, "%d sequences, the cache has room for %d", n_new, kv->max_seqs);
    if ((n_new && !parent) || !status) return bad(SDLM_EINVAL, "parent and status are required");
    if ((rc = check_workspace(workspace, bytes, fork_workspace_bytes(*kv)))) return rc;
    launch_fork((hipStream_t)hip_stream, *kv, parent, n_new, share != 0, status, workspace);
    return launched("sdlm_kv_fork");
}

int sdlm_kv_compact(const sdlm_kv *kv, int32_t n_seqs, const int32_t *path, int32_t path_stride, const int32_t *path_len, int32_t max_path, const int32_t *node_table,
                    int32_t node_pages, const int32_t *node_base, void *hip_stream)
{
    const int rc = check_kv(kv, false);
    if (rc) return rc;
    if (n_seqs < 0 || n_seqs > kv->max_seqs || n_seqs > 65535) return bad(SDLM_EINVAL, "%d sequences, the cache has %d (at most 65535 in a call)", n_seqs, kv->max_seqs);
    if (max_path < 0 || path_stride < max_path || node_pages < 1 || node_pages > MAX_TABLE)
        return bad(SDLM_EINVAL, "path_stride must hold max_path >= 0 nodes, and node_pages be 1 .. %d", MAX_TABLE);
    if (n_seqs == 0 || max_path == 0) return SDLM_OK;
    if (!path || !path_len || !node_table) return bad(SDLM_EINVAL, "path, path_len and node_table are required");
    launch_compact((hipStream_t)hip_stream, *kv, kv->lengths, node_table, node_pages, node_base, path, path_stride, path_len, n_seqs, max_path);
    return launched("sdlm_kv_compact");
}

}  // extern "C"
