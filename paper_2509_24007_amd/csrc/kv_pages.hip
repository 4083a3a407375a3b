// Pages of a K/V cache: forking sequences (sharing, copying and freeing their pages) and moving single positions.
//
// A page that is full never changes again, so sequences that start alike share it; what is still being written belongs to one
// sequence.  page_refs counts the sequences that hold a page, and a page that nobody holds is free.  Nothing here computes: the
// bookkeeping is integers whose result does not depend on the order of the threads, and the K/V are copied bit for bit.
#include "ops.hpp"

namespace sdlm {

namespace {

struct ForkWs {
    int32_t *table, *len, *held;   // the sequences as they were
    int32_t *refs;                 // [n_pages] holders after the fork, new pages not counted yet
    int32_t *free_list;            // [n_pages] pages without a holder, ascending
    int32_t *src;                  // [n_pages] what the i-th of them receives: the page that it is a copy of, -1: nothing
    int32_t *first, *fresh;        // [max_seqs + 1] first new page of a new sequence (its index in free_list), first position that is not shared
    int32_t *head;                 // [4] new pages handed out (0 if the fork is refused), free pages, problems found
};

struct ForkArgs {
    sdlm_kv kv;
    const int32_t *parent;
    int32_t *status;
    int n_new, share;
    ForkWs w;
};

size_t up(size_t v) { return (v + 255) / 256 * 256; }

ForkWs fork_ws(const sdlm_kv &kv, void *workspace, size_t *bytes)
{
    char *p = (char *)workspace;
    size_t o = 0;
    auto take = [&](size_t n) { int32_t *at = (int32_t *)(p + o); o += up(n * sizeof(int32_t)); return at; };
    ForkWs w;
    w.table = take((size_t)kv.max_seqs * kv.pages_per_seq);
    w.len = take(kv.max_seqs); w.held = take(kv.max_seqs);
    w.refs = take(kv.n_pages); w.free_list = take(kv.n_pages); w.src = take(kv.n_pages);
    w.first = take(kv.max_seqs + 1); w.fresh = take(kv.max_seqs);
    w.head = take(4);
    *bytes = o;
    return w;
}

// 1: the old state is set aside, since a new sequence's entries may overwrite those that another one still reads.
__global__ __launch_bounds__(256) void fork_save_k(ForkArgs a)
{
    const long n = (long)a.kv.max_seqs * a.kv.pages_per_seq, step = (long)gridDim.x * 256, t0 = (long)blockIdx.x * 256 + threadIdx.x;
    for (long i = t0; i < n; i += step) a.w.table[i] = a.kv.page_table[i];
    for (long i = t0; i < a.kv.n_pages; i += step) a.w.refs[i] = 0;
    for (long i = t0; i < a.kv.max_seqs; i += step) {
        const int held = min(max(a.kv.backed[i], 0), a.kv.pages_per_seq);
        a.w.held[i] = held;
        a.w.len[i] = min(max(a.kv.lengths[i], 0), held * PAGE);
    }
    if (t0 < 4) a.w.head[t0] = 0;
}

// 2: one workgroup a new sequence: whether it inherits its parent's own pages, and one more holder for every page that it takes over.
__global__ __launch_bounds__(256) void fork_count_k(ForkArgs a)
{
    const int b = blockIdx.x, p = a.parent[b];
    if (p < -1 || p >= a.kv.max_seqs) {
        if (threadIdx.x == 0) { atomicOr(&a.w.head[2], 2); a.w.fresh[b] = 0; a.w.first[b] = 0; }
        return;
    }
    // The parent's own pages stay with it, or, if it ends here, go to the first of its children.
    const bool stays = p >= 0 && p < a.n_new && a.parent[p] == p;
    bool earlier = false;
    if (p >= 0 && !stays)
        for (int i = threadIdx.x; i < b; i += 256) earlier |= a.parent[i] == p;
    const bool heir = p >= 0 && (stays ? b == p : !__syncthreads_or(earlier));
    const int held = p < 0 ? 0 : a.w.held[p], shared = p < 0 ? 0 : a.share ? a.w.len[p] / PAGE : 0, keep = heir ? held : shared;
    if (threadIdx.x == 0) { a.w.fresh[b] = keep; a.w.first[b] = held - keep; }   // first: a count as yet
    for (int j = threadIdx.x; j < held; j += 256) {
        const int page = a.w.table[(size_t)p * a.kv.pages_per_seq + j];
        if (page < 0 || page >= a.kv.n_pages) atomicOr(&a.w.head[2], 2);
        else if (j < keep) atomicAdd(&a.w.refs[page], 1);
    }
}

// Exclusive prefix sum over the threads of a workgroup of 1024; total: the sum.
__device__ inline int block_scan(int v, int *total)
{
    __shared__ int part[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
    for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(x, o); if (lane >= o) x += y; }
    __syncthreads();
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int before = 0, sum = 0;
    for (int w = 0; w < 16; ++w) { if (w < wave) before += part[w]; sum += part[w]; }
    *total = sum;
    return before + x - v;
}

// 3: one workgroup: the list of free pages, and where in it each new sequence's new pages begin.
__global__ __launch_bounds__(1024) void fork_plan_k(ForkArgs a)
{
    int n_free = 0, need = 0, sum;
    for (int p0 = 0; p0 < a.kv.n_pages; p0 += 1024) {
        const int p = p0 + threadIdx.x;
        const int is_free = p < a.kv.n_pages && a.w.refs[p] == 0;
        const int at = n_free + block_scan(is_free, &sum);
        if (is_free) a.w.free_list[at] = p;
        n_free += sum;
    }
    for (int b0 = 0; b0 < a.n_new; b0 += 1024) {
        const int b = b0 + threadIdx.x, v = b < a.n_new ? a.w.first[b] : 0;
        const int at = need + block_scan(v, &sum);
        if (b < a.n_new) a.w.first[b] = at;
        need += sum;
    }
    if (threadIdx.x == 0) {
        int bad = a.w.head[2];
        if (need > n_free) bad |= 1;
        a.w.first[a.n_new] = need;
        a.w.head[0] = bad ? 0 : need;
        a.w.head[1] = n_free;
        a.w.head[2] = bad;
        *a.status = bad;
    }
}

// 4: the new tables, lengths, counts and free list (left as they are if the fork is refused).
__global__ __launch_bounds__(256) void fork_write_k(ForkArgs a)
{
    if (a.w.head[2]) return;
    const int need = a.w.head[0], n_free = a.w.head[1];
    const int b = blockIdx.x, pps = a.kv.pages_per_seq;
    if (b < a.kv.max_seqs) {
        const int p = b < a.n_new ? a.parent[b] : -1, held = p < 0 ? 0 : a.w.held[p], len = p < 0 ? 0 : a.w.len[p];
        const int fresh = p < 0 ? 0 : a.w.fresh[b], first = p < 0 ? 0 : a.w.first[b];
        for (int j = threadIdx.x; j < pps; j += 256) {
            int page = -1;
            if (j < held) {
                page = a.w.table[(size_t)p * pps + j];
                if (j >= fresh) {
                    const int i = first + j - fresh;
                    a.w.src[i] = j * PAGE < len ? page : -1;   // pages behind the end have nothing to copy
                    page = a.w.free_list[i];
                }
            }
            a.kv.page_table[(size_t)b * pps + j] = page;
        }
        if (threadIdx.x == 0) { a.kv.lengths[b] = len; a.kv.backed[b] = held; }
    }
    const long step = (long)gridDim.x * 256;
    for (long i = (long)b * 256 + threadIdx.x; i < a.kv.n_pages; i += step) {
        const bool is_free = i < n_free;
        const int p = is_free ? a.w.free_list[i] : 0;
        a.kv.free_pages[i] = i + need < n_free ? a.w.free_list[i + need] : -1;
        if (is_free) a.kv.page_refs[p] = i < need ? 1 : 0;
        const int r = a.w.refs[i];
        if (r) a.kv.page_refs[i] = r;
    }
    if (b == 0 && threadIdx.x == 0) *a.kv.free_count = n_free - need;
}

// 1 to 4 in one workgroup, for caches whose tables fit LDS: the launches in front of the copies are most of a fork's time (us a fork, 64 sequences of 258 pages 21.8 -> 12.4, 5 of 9 pages 20.6 -> 11.8).
constexpr int SMALL_TABLE = 20480, SMALL_PAGES = 12288, SMALL_SEQS = 512;

bool fork_small(const sdlm_kv &kv) { return (long)kv.max_seqs * kv.pages_per_seq <= SMALL_TABLE && kv.n_pages <= SMALL_PAGES && kv.max_seqs <= SMALL_SEQS; }

__global__ __launch_bounds__(1024) void fork_small_k(ForkArgs a)
{
    __shared__ int32_t table[SMALL_TABLE], refs[SMALL_PAGES];
    __shared__ int32_t len[SMALL_SEQS], held[SMALL_SEQS], par[SMALL_SEQS], heir[SMALL_SEQS], keep[SMALL_SEQS], first[SMALL_SEQS];
    __shared__ int bad_s;
    const int tid = threadIdx.x, S = a.kv.max_seqs, pps = a.kv.pages_per_seq, P = a.kv.n_pages;
    for (int i = tid; i < S * pps; i += 1024) table[i] = a.kv.page_table[i];
    for (int i = tid; i < P; i += 1024) refs[i] = 0;
    if (tid == 0) bad_s = 0;
    if (tid < S) {
        const int h = min(max(a.kv.backed[tid], 0), pps), p = tid < a.n_new ? a.parent[tid] : -1;
        held[tid] = h;
        len[tid] = min(max(a.kv.lengths[tid], 0), h * PAGE);
        par[tid] = p;
        heir[tid] = S;
    }
    __syncthreads();
    const int p = tid < S ? par[tid] : -1;
    const bool in = p >= 0 && p < S;
    if (p < -1 || p >= S) bad_s = 2;
    if (in) atomicMin(&heir[p], tid);   // its first child
    __syncthreads();
    int fresh = 0;
    if (tid < S) {
        // the parent's own pages stay with it, or, if it ends here, go to the first of its children
        const bool mine = in && (p < a.n_new && par[p] == p ? tid == p : heir[p] == tid);
        keep[tid] = !in ? 0 : mine ? held[p] : a.share ? len[p] / PAGE : 0;
        fresh = in ? held[p] - keep[tid] : 0;
    }
    __syncthreads();
    const int wave = tid >> 6, lane = tid & 63;   // a wavefront a sequence
    for (int b = wave; b < a.n_new; b += 16) {
        const int q = par[b];
        if (q < 0 || q >= S) continue;
        const int h = held[q], own = keep[b];
        for (int j = lane; j < h; j += 64) {
            const int page = table[q * pps + j];
            if (page < 0 || page >= P) bad_s = 2;
            else if (j < own) atomicAdd(&refs[page], 1);
        }
    }
    __syncthreads();
    // free pages: a stretch of them a thread
    const int per = (P + 1023) / 1024, p0 = min(tid * per, P), p1 = min(p0 + per, P);
    int mine_free = 0, n_free, need;
    for (int i = p0; i < p1; ++i) mine_free += refs[i] == 0;
    int at = block_scan(mine_free, &n_free);
    const int at_new = block_scan(fresh, &need);
    if (tid < S) first[tid] = at_new;
    const int bad = bad_s | (need > n_free ? 1 : 0);
    if (tid == 0) { a.w.head[0] = bad ? 0 : need; *a.status = bad; }
    if (bad) return;
    for (int i = p0; i < p1; ++i) {
        int r = refs[i];
        if (r == 0) {
            if (at < need) { a.w.free_list[at] = i; r = 1; }
            else a.kv.free_pages[at - need] = i;
            ++at;
        }
        a.kv.page_refs[i] = r;
    }
    for (int i = n_free - need + tid; i < P; i += 1024) a.kv.free_pages[i] = -1;
    if (tid == 0) *a.kv.free_count = n_free - need;
    __threadfence_block();
    __syncthreads();
    for (int b = wave; b < S; b += 16) {
        const int q = par[b], h = q < 0 ? 0 : held[q], own = keep[b], k0 = first[b] - own, n = q < 0 ? 0 : len[q];
        for (int j = lane; j < pps; j += 64) {
            int page = -1;
            if (j < h) {
                page = table[q * pps + j];
                if (j >= own) {
                    a.w.src[k0 + j] = j * PAGE < n ? page : -1;   // pages behind the end have nothing to copy
                    page = a.w.free_list[k0 + j];
                }
            }
            a.kv.page_table[b * pps + j] = page;
        }
    }
    if (tid < S) { a.kv.lengths[tid] = in ? len[p] : 0; a.kv.backed[tid] = in ? held[p] : 0; }
}

// 5: the copies, 16 bytes a thread at a time: unit = one (new page, layer), consecutive in the pool.  Bound by memory: 100 MB in 40 us (5.0 TB/s read and written).
__global__ __launch_bounds__(256) void fork_copy_k(ForkArgs a, int vec_per_page, size_t layer_vecs)
{
    const long units = (long)a.w.head[0] * a.kv.n_layers;
    uint4 *pool = (uint4 *)a.kv.pool;
    for (long u = blockIdx.x; u < units; u += gridDim.x) {
        const int i = (int)(u / a.kv.n_layers), l = (int)(u % a.kv.n_layers), src = a.w.src[i];
        if (src < 0) continue;
        const uint4 *from = pool + l * layer_vecs + (size_t)src * vec_per_page;
        uint4 *to = pool + l * layer_vecs + (size_t)a.w.free_list[i] * vec_per_page;
        for (int e = threadIdx.x; e < vec_per_page; e += 256) to[e] = from[e];
    }
}

}  // namespace

size_t fork_workspace_bytes(const sdlm_kv &kv)
{
    size_t n;
    fork_ws(kv, nullptr, &n);
    return n;
}

void launch_fork(hipStream_t s, const sdlm_kv &kv, const int32_t *parent, int n_new, int share, int32_t *status, void *workspace)
{
    ForkArgs a;
    size_t n;
    a.kv = kv; a.parent = parent; a.status = status; a.n_new = n_new; a.share = share;
    a.w = fork_ws(kv, workspace, &n);
    const size_t esz = kv.dtype == 0 ? 4 : 2;
    const int vec_per_page = (int)((size_t)kv.n_kv_heads * 2 * PAGE * kv.head_dim * esz / 16);
    if (fork_small(kv)) hipLaunchKernelGGL(fork_small_k, dim3(1), dim3(1024), 0, s, a);
    else {
        hipLaunchKernelGGL(fork_save_k, dim3(512), dim3(256), 0, s, a);
        if (n_new > 0) hipLaunchKernelGGL(fork_count_k, dim3(n_new), dim3(256), 0, s, a);
        hipLaunchKernelGGL(fork_plan_k, dim3(1), dim3(1024), 0, s, a);
        hipLaunchKernelGGL(fork_write_k, dim3(kv.max_seqs), dim3(256), 0, s, a);
    }
    const long units = (long)n_new * (share ? 1 : kv.pages_per_seq) * kv.n_layers;   // share: at most the page that is being written has contents
    if (n_new > 0) hipLaunchKernelGGL(fork_copy_k, dim3(units < 2048 ? units : 2048), dim3(256), 0, s, a, vec_per_page, (size_t)kv.layer_stride * esz / 16);
}

namespace {

// K/V of the nodes path[b][0 .. g) -> positions start[b] .. start[b] + g - 1 of sequence b.  One workgroup a (sequence, layer, kv head): it reads MOVE positions before it
// writes any, and a path ascends (path[i] >= i), so the nodes may stand behind the sequence in its own pages.  A thread an element of a position: K is in pieces of
// 16 bytes, V in single elements all over the tile.  Bound by its chain of round trips (length, path, tables, elements): one lane a position looks up both places (us:
// 4 nodes of one sequence, 28 layers 4.4; 64 sequences, 14 layers, 4 heads, up to 5 nodes 12).
constexpr int MOVE = 8;

template <typename T>
__global__ __launch_bounds__(256) void compact_k(sdlm_kv kv, const int32_t *start, const int32_t *node_table, int node_pages, const int32_t *node_base, const int32_t *path,
                                                 int path_stride, const int32_t *path_len, int max_path)
{
    const int b = blockIdx.y, l = blockIdx.x / kv.n_kv_heads, h = blockIdx.x % kv.n_kv_heads, d = kv.head_dim, tid = threadIdx.x;
    const int g = min(path_len[b], max_path), s0 = start[b], base = node_base ? node_base[b] : 0;
    T *pool = (T *)kv.pool + (size_t)l * kv.layer_stride;
    const size_t tile = (size_t)2 * PAGE * d;
    __shared__ int2 place[2][MOVE];   // [from, to]: page (-1: passed over) and slot
    const int e = tid < d ? tid : tid - d;
    const bool k = tid < d, on = tid < 2 * d;
    auto at = [&](const int2 &p) { return pool + ((size_t)p.x * kv.n_kv_heads + h) * tile + (k ? k_off(p.y, e) : PAGE * d + v_off(p.y, e)); };
    for (int m0 = 0; m0 < g; m0 += MOVE) {
        if (tid < MOVE) {
            int2 from = make_int2(-1, 0), to = from;
            if (m0 + tid < g) {
                const int node = path[(size_t)b * path_stride + m0 + tid];
                const long src = (long)base + node, dst = (long)s0 + m0 + tid;
                if (node >= 0 && src >= 0 && src / PAGE < node_pages && dst >= 0 && dst / PAGE < kv.pages_per_seq) {
                    const int a = node_table[(size_t)b * node_pages + src / PAGE], c = kv.page_table[(size_t)b * kv.pages_per_seq + dst / PAGE];
                    if (a >= 0 && a < kv.n_tiles && c >= 0 && c < kv.n_tiles) { from = make_int2(a, (int)(src % PAGE)); to = make_int2(c, (int)(dst % PAGE)); }
                }
            }
            place[0][tid] = from;
            place[1][tid] = to;
        }
        __syncthreads();
        T v[MOVE];
#pragma unroll
        for (int q = 0; q < MOVE; ++q) {
            v[q] = T(0);
            if (on && place[0][q].x >= 0) v[q] = *at(place[0][q]);
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < MOVE; ++q)
            if (on && place[1][q].x >= 0) *at(place[1][q]) = v[q];
        __syncthreads();   // places, and positions that the next nodes may stand behind
    }
}

}  // namespace

void launch_compact(hipStream_t s, const sdlm_kv &kv, const int32_t *start, const int32_t *node_table, int node_pages, const int32_t *node_base, const int32_t *path,
                    int path_stride, const int32_t *path_len, int n_seqs, int max_path)
{
    const dim3 grid(kv.n_layers * kv.n_kv_heads, n_seqs);
    if (kv.dtype == 0) hipLaunchKernelGGL(compact_k<float>, grid, dim3(256), 0, s, kv, start, node_table, node_pages, node_base, path, path_stride, path_len, max_path);
    else hipLaunchKernelGGL(compact_k<bf16_t>, grid, dim3(256), 0, s, kv, start, node_table, node_pages, node_base, path, path_stride, path_len, max_path);
}

}  // namespace sdlm
