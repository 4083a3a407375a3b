// Attention of drafted token trees over a K/V cache: every node of a sequence sees the sequence's first `length` positions, and of the nodes
// those that its mask names.
//   out[r, h] = sum_j p_j V[j], p = softmax over the seen keys of q[r, h] . K[j] / sqrt(d); a node that sees no key gets zeros.
#include <math.h>

#include "ops.hpp"

namespace sdlm {

namespace {

struct TreeArgs {
    sdlm_kv kv;
    sdlm_tree_args t;
    const void *pool;   // this layer's tiles
    float scale;
};

// One wavefront a (node, query head), a key a lane; a running maximum, sum and output.
template <typename T, int HD>
__global__ __launch_bounds__(64) void tree_rows_k(TreeArgs a)
{
    constexpr int FD = (HD + 63) / 64;
    const int r = blockIdx.y, hq = blockIdx.x, lane = threadIdx.x, G = a.t.n_q_heads / a.kv.n_kv_heads, hk = hq / G;
    int b = -1;   // the sequence whose nodes include r
    for (int i = lane; i < a.t.n_seqs; i += 64)
        if (r >= a.t.node_offsets[i] && r < a.t.node_offsets[i + 1]) b = i;
    for (int o = 32; o > 0; o >>= 1) b = max(b, __shfl_xor(b, o));
    if (b < 0) return;
    const int first = a.t.node_offsets[b], nodes = min(a.t.node_offsets[b + 1] - first, a.t.max_nodes);
    if (r - first >= nodes) return;
    const int len = min(max(a.kv.lengths[b], 0), a.kv.pages_per_seq * PAGE), base = a.t.node_base ? a.t.node_base[b] : 0;
    const u_int64_t *mask = (const u_int64_t *)a.t.mask + (size_t)r * a.t.mask_words;
    const size_t tile = (size_t)2 * PAGE * HD;
    const T *pool = (const T *)a.pool;
    __shared__ float q[HD];
    for (int i = lane; i < HD; i += 64) q[i] = to_f<T>(((const T *)a.t.q)[(size_t)r * a.t.q_stride + hq * HD + i]) * a.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[FD] = {};
    for (int j0 = 0; j0 < len + nodes; j0 += 64) {
        const int j = j0 + lane;
        int page = -1, slot = 0;
        if (j < len) { page = a.kv.page_table[(size_t)b * a.kv.pages_per_seq + j / PAGE]; slot = j % PAGE; }
        else if (j < len + nodes) {
            const int n = j - len, at = base + n;
            if (((mask[n >> 6] >> (n & 63)) & 1) && at >= 0 && at / PAGE < a.t.node_pages) { page = a.t.node_table[(size_t)b * a.t.node_pages + at / PAGE]; slot = at % PAGE; }
        }
        if (page >= a.kv.n_tiles) page = -1;
        const T *t = pool + ((size_t)max(page, 0) * a.kv.n_kv_heads + hk) * tile;
        float s = -INFINITY;
        if (page >= 0) {
            s = 0.f;
            for (int i = 0; i < HD; ++i) s += q[i] * to_f<T>(t[k_off(slot, i)]);
        }
        float mx = s;
        for (int d = 32; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
        const float mn = fmaxf(m, mx), corr = m == -INFINITY ? 0.f : __expf(m - mn), p = page < 0 ? 0.f : __expf(s - mn);
        m = mn;
        l = l * corr + p;
        for (int f = 0; f < FD; ++f) o[f] *= corr;
        for (int k = 0; k < 64; ++k) {
            const int pk = __shfl(page, k), sk = __shfl(slot, k);
            const float w = __shfl(p, k);
            if (pk < 0) continue;
            const T *v = pool + ((size_t)pk * a.kv.n_kv_heads + hk) * tile + PAGE * HD;
            for (int f = 0; f < FD; ++f)
                if (lane + 64 * f < HD) o[f] += w * to_f<T>(v[v_off(sk, lane + 64 * f)]);
        }
    }
    for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
    for (int f = 0; f < FD; ++f)
        if (lane + 64 * f < HD) ((T *)a.t.out)[(size_t)r * a.t.out_stride + hq * HD + lane + 64 * f] = from_f<T>(m == -INFINITY ? 0.f : o[f] / l);
}

template <typename T>
void rows_t(hipStream_t s, const TreeArgs &a)
{
    const dim3 grid(a.t.n_q_heads, a.t.n_rows), block(64);
    switch (a.kv.head_dim) {
    case 32: hipLaunchKernelGGL((tree_rows_k<T, 32>), grid, block, 0, s, a); break;
    case 64: hipLaunchKernelGGL((tree_rows_k<T, 64>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((tree_rows_k<T, 96>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((tree_rows_k<T, 128>), grid, block, 0, s, a); break;
    }
}

}  // namespace

size_t tree_workspace_bytes(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes, int max_len) { return 256; }

void launch_tree_attention(hipStream_t s, const sdlm_kv &kv, int layer, const sdlm_tree_args &t, void *workspace, size_t workspace_bytes)
{
    TreeArgs a;
    a.kv = kv; a.t = t;
    a.pool = (const char *)kv.pool + (size_t)layer * kv.layer_stride * (kv.dtype == 0 ? 4 : 2);
    a.scale = 1.0f / sqrtf((float)kv.head_dim);
    if (kv.dtype == 0) rows_t<float>(s, a); else rows_t<bf16_t>(s, a);
}

}  // namespace sdlm
