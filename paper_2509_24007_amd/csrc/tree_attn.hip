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

// ------------------------------------------------------------------------------------------------ matrix-core path (bf16)
// A work item is (sequence, block of queries, run of tiles, kv head): its queries are the (node, query head) pairs that read the kv head, 16 QT for each of four
// wavefronts, and all of them use every tile that the workgroup brings to LDS.  The items of a launch are laid out on the device from the actual lengths: every
// wavefront reads the lengths and offsets of all sequences (a lane a sequence) and finds its own item by prefix sums, so ragged batches need no plan launch.
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
union Op8 { bf16x8 v; uint4 u; uint2 h[2]; uint32_t w[4]; };

constexpr int ITEMS = 512;            // work items to aim at, over all kv heads
constexpr int MIN_TILES = 4;          // fewest tiles of an item, where a sequence has that many
constexpr float RESCALE_GAP = 8.0f;   // log2 units, see the running maximum below

__device__ inline bool finite16(uint32_t x) { return (x & 0x7f80u) != 0x7f80u; }   // of a bf16's bits

struct MfmaArgs {
    TreeArgs t;
    float *part_o;      // [item][kv head][query of the block][HD]
    float2 *part_ml;    // [item][kv head][query of the block]: running maximum, sum
    float c;            // log2(e) / sqrt(d)
    int G;
};

struct Seq { int first, nodes, len, base, prefix_tiles, tiles, blocks; };

__device__ inline Seq seq_of(const TreeArgs &a, int b, int G, int qb)
{
    Seq s;
    s.first = min(max(a.t.node_offsets[b], 0), a.t.n_rows);
    s.nodes = min(max(min(a.t.node_offsets[b + 1], a.t.n_rows) - s.first, 0), a.t.max_nodes);
    s.len = min(max(a.kv.lengths[b], 0), a.kv.pages_per_seq * PAGE);
    s.base = a.t.node_base ? min(max(a.t.node_base[b], 0), a.t.node_pages * PAGE) : 0;
    s.prefix_tiles = (s.len + PAGE - 1) / PAGE;
    s.tiles = s.prefix_tiles + (s.base % PAGE + s.nodes + PAGE - 1) / PAGE;
    s.blocks = (s.nodes * G + qb - 1) / qb;
    return s;
}

// Tiles of an item: as many as leave about ITEMS items, an even number.
__device__ inline int item_tiles(long all_tiles, int n_kv_heads)
{
    const long per = (all_tiles * n_kv_heads + ITEMS - 1) / ITEMS;
    return (int)max((per + 1) / 2 * 2, (long)MIN_TILES);
}

// The sequence b, and the number of its first item, that item `want` belongs to (b = -1: there is no such item).  merge: counts blocks instead of items; `before` is then
// the first block's number and `item0` its sequence's first item.
struct Place { int b, before, item0, cp; };

__device__ inline Place place_of(const TreeArgs &a, int G, int qb, int want, bool merge)
{
    const int lane = threadIdx.x & 63, S = a.t.n_seqs;
    long all = 0;
    for (int b0 = 0; b0 < S; b0 += 64) {
        if (b0 + lane < S) { const Seq s = seq_of(a, b0 + lane, G, qb); all += (long)s.blocks * s.tiles; }
    }
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o);
    Place p{-1, 0, 0, item_tiles(all, a.kv.n_kv_heads)};
    int items = 0, blocks = 0;
    for (int b0 = 0; b0 < S; b0 += 64) {
        int n = 0, nb = 0;
        if (b0 + lane < S) {
            const Seq s = seq_of(a, b0 + lane, G, qb);
            nb = s.blocks;
            n = nb * ((s.tiles + p.cp - 1) / p.cp);
        }
        int xi = n, xb = nb;
        for (int o = 1; o < 64; o <<= 1) {
            const int yi = __shfl_up(xi, o), yb = __shfl_up(xb, o);
            if (lane >= o) { xi += yi; xb += yb; }
        }
        const int end = merge ? blocks + xb : items + xi;
        const uint64_t past = __ballot(want < end);   // the first lane whose items end behind `want`
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            p.b = b0 + at;
            p.item0 = __shfl(items + xi - n, at);
            p.before = merge ? __shfl(blocks + xb - nb, at) : p.item0;
            return p;
        }
        items += __shfl(xi, 63);
        blocks += __shfl(xb, 63);
    }
    return p;
}

template <int HD, int QT>
__global__ __launch_bounds__(256, QT == 1 ? 4 : 2) void tree_mfma_k(MfmaArgs a)
{
    constexpr int QB = 64 * QT, NK = HD / 32, ND = HD / 16, TILE = 2 * PAGE * HD, VEC = HD / 32;   // VEC: 16-byte loads of a thread for a pair of tiles
    const int hk = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, lg = lane >> 4, G = a.G;
    Place pl = place_of(a.t, G, QB, blockIdx.x, false);
    const int b = __builtin_amdgcn_readfirstlane(pl.b);
    if (b < 0) return;
    const int cp = __builtin_amdgcn_readfirstlane(pl.cp);
    const Seq s = seq_of(a.t, b, G, QB);
    const int local = blockIdx.x - __builtin_amdgcn_readfirstlane(pl.item0), block = local % s.blocks, chunk = local / s.blocks;
    const int u0 = chunk * cp, u1 = min(s.tiles, u0 + cp), n_pairs = (u1 - u0 + 1) / 2, n_chunks = (s.tiles + cp - 1) / cp;
    const int q0 = block * QB + wave * 16 * QT, QR = s.nodes * G;
    const bool active = q0 < QR;
    const int32_t *ptab = a.t.kv.page_table + (size_t)b * a.t.kv.pages_per_seq, *ntab = a.t.t.node_table + (size_t)b * a.t.t.node_pages;
    const int node_tile0 = s.base / PAGE - s.prefix_tiles, shift0 = s.prefix_tiles * PAGE + s.base % PAGE;   // tile u >= prefix_tiles: entry u + node_tile0; its slot i is node u 16 + i - shift0

    Op8 qop[QT][NK];
    int mrow[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int qi = q0 + t * 16 + ln;
        const bool ok = qi < QR;
        const int row = s.first + (ok ? qi / G : 0), h = hk * G + (ok ? qi % G : 0);
        const bf16_t *qp = (const bf16_t *)a.t.t.q + (size_t)row * a.t.t.q_stride + h * HD + lg * 8;
        mrow[t] = row;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            qop[t][kk].u = make_uint4(0, 0, 0, 0);
            if (ok) qop[t][kk].u = *(const uint4 *)(qp + kk * 32);
        }
    }
    f32x4 O[QT][ND];
    float m_run[QT], l_run[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m_run[t] = -INFINITY; l_run[t] = 0.f;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) O[t][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    __shared__ __attribute__((aligned(16))) bf16_t kv[2][2 * TILE];   // two pairs of tiles, each as in the pool
    const bf16_t *pool = (const bf16_t *)a.t.pool;
    // page of tile u, -1 where there is none
    auto page = [&](int u) -> int {
        if (u >= u1) return -1;
        int p = -1;
        if (u < s.prefix_tiles) p = ptab[u];
        else if (u + node_tile0 < a.t.t.node_pages) p = ntab[u + node_tile0];
        return p < a.t.kv.n_tiles ? p : -1;
    };
    // a pair in flight: its tiles' contents, and whether they exist
    auto fetch = [&](int pp, u32x4 (&r)[VEC]) -> int {
        const int pA = page(u0 + 2 * pp), pB = page(u0 + 2 * pp + 1);
        const bf16_t *tA = pool + ((size_t)max(pA, 0) * a.t.kv.n_kv_heads + hk) * TILE, *tB = pool + ((size_t)max(pB >= 0 ? pB : pA, 0) * a.t.kv.n_kv_heads + hk) * TILE;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int e = tid + 256 * i;
            r[i] = *(const u32x4 *)((e < TILE / 8 ? tA : tB - TILE) + (size_t)e * 8);
        }
        return (pA >= 0 ? 1 : 0) | (pB >= 0 ? 2 : 0);
    };
    __shared__ int strange[2][4];   // per wavefront: whether its part of the pair's values has some that are not finite (only where a query may not see all slots)
    auto is_whole = [&](int pp, int have) { return have == 3 && (u0 + 2 * pp + 2) * PAGE <= s.len; };   // every key of the pair is seen by every query
    auto stash = [&](int buf, const u32x4 (&r)[VEC], int pp, int have) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) *(u32x4 *)(&kv[buf][0] + (size_t)(tid + 256 * i) * 8) = r[i];
        if (is_whole(pp, have)) return;
        bool any = false;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if ((tid + 256 * i) % (TILE / 8) >= TILE / 16)
#pragma unroll
                for (int k = 0; k < 4; ++k) any |= !finite16(r[i][k]) || !finite16(r[i][k] >> 16);
        any = __any(any);
        if (lane == 0) strange[buf][wave] = any;
    };
    auto compute = [&](int pp, int buf, int have) {
        if (!active) return;
        const int uA = u0 + 2 * pp;
        const bf16_t *KA = &kv[buf][0], *KB = KA + TILE;
        f32x4 sA[QT], sB[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) { sA[t] = f32x4{0.f, 0.f, 0.f, 0.f}; sB[t] = sA[t]; }
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            Op8 ka, kb;
            ka.u = *(const uint4 *)(KA + (kk * 64 + lane) * 8);
            kb.u = *(const uint4 *)(KB + (kk * 64 + lane) * 8);
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                sA[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka.v, qop[t][kk].v, sA[t], 0, 0, 0);
                sB[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb.v, qop[t][kk].v, sB[t], 0, 0, 0);
            }
        }
        const bool whole = is_whole(pp, have);
        uint32_t seen[QT];   // bits 0..15: slots of tile A that the query sees, 16..31: of tile B
        if (!whole) {
            const int left = s.len - uA * PAGE;   // positions of the prefix in the pair; what is above are slots behind its end, or nodes
            const uint32_t pre = left <= 0 ? 0u : left >= 32 ? ~0u : (1u << left) - 1u;
            const uint32_t exist = (have & 1 ? 0xffffu : 0u) | (have & 2 ? 0xffff0000u : 0u);
            const uint32_t is_node = uA >= s.prefix_tiles ? ~0u : uA + 1 >= s.prefix_tiles ? 0xffff0000u : 0u;
            const int at = uA * PAGE - shift0;    // node of the pair's first slot (may be negative)
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                seen[t] = pre & ~is_node;
                if (is_node) {
                    const int w = at > 0 ? at >> 6 : 0, sh = at > 0 ? at & 63 : 0;
                    const int64_t *words = a.t.t.mask + (size_t)mrow[t] * a.t.t.mask_words;
                    uint64_t bits = 0;
                    if (w < a.t.t.mask_words) bits = (uint64_t)words[w] >> sh;
                    if (sh && w + 1 < a.t.t.mask_words) bits |= (uint64_t)words[w + 1] << (64 - sh);
                    if (at < 0) bits <<= -at;
                    const int n = s.nodes - at;   // slots up to the last node
                    seen[t] |= (uint32_t)bits & (n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u) & is_node;
                }
                seen[t] &= exist;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    sA[t][v] = (seen[t] >> (lg * 4 + v)) & 1u ? sA[t][v] : -INFINITY;
                    sB[t][v] = (seen[t] >> (16 + lg * 4 + v)) & 1u ? sB[t][v] : -INFINITY;
                }
            }
        }
        Op8 pop[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            // raw scores; the softmax scale is folded into the exponent: p = 2^(c s - c m).  The reference maximum only moves when it is exceeded by more than
            // RESCALE_GAP / c (p stays below 2^RESCALE_GAP, harmless in fp32 sums and bf16 products); the accumulators are rescaled only then.
            float mx = fmaxf(fmaxf(fmaxf(sA[t][0], sA[t][1]), fmaxf(sA[t][2], sA[t][3])), fmaxf(fmaxf(sB[t][0], sB[t][1]), fmaxf(sB[t][2], sB[t][3])));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            if (__any((mx - m_run[t]) * a.c > RESCALE_GAP || (m_run[t] == -INFINITY && mx > -INFINITY))) {
                const float m_new = fmaxf(m_run[t], mx);
                const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run[t] - m_new) * a.c);
                l_run[t] *= corr;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) O[t][dt] *= corr;
                m_run[t] = m_new;
            }
            const float mc = m_run[t] == -INFINITY ? 0.f : m_run[t] * a.c;
            float p[8];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                p[v] = __builtin_amdgcn_exp2f(fmaf(sA[t][v], a.c, -mc));
                p[4 + v] = __builtin_amdgcn_exp2f(fmaf(sB[t][v], a.c, -mc));
            }
            l_run[t] += (p[0] + p[1]) + (p[2] + p[3]) + (p[4] + p[5]) + (p[6] + p[7]);
            pop[t].w[0] = pack_bf16(p[0], p[1]); pop[t].w[1] = pack_bf16(p[2], p[3]);
            pop[t].w[2] = pack_bf16(p[4], p[5]); pop[t].w[3] = pack_bf16(p[6], p[7]);
        }
        const bf16_t *VA = KA + PAGE * HD, *VB = KB + PAGE * HD;
        // A slot that a query does not see may hold anything, and 0 times a value that is not finite is not 0.  Such values are added one by one for the queries that see them.
        const bool odd = !whole && (strange[buf][0] | strange[buf][1] | strange[buf][2] | strange[buf][3]);
        if (odd) {
#pragma unroll 1
            for (int slot = 0; slot < 32; ++slot) {
                const int k = (slot >> 4) * 2 + ((slot & 3) >> 1), from = (slot >> 2 & 3) * 16 + ln;   // the word and the lane of the query's weight for this slot
                const bf16_t *Vs = (slot < 16 ? VA : VB) + ((slot >> 2 & 3) * 16 + lg * 4) * 4 + (slot & 3);
                float w[QT];
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    const uint32_t lo = k & 1 ? pop[t].w[1] : pop[t].w[0], hi = k & 1 ? pop[t].w[3] : pop[t].w[2], mine = k & 2 ? hi : lo;
                    const uint32_t x = (uint32_t)__shfl((int)mine, from);
                    w[t] = __uint_as_float(slot & 1 ? x & 0xffff0000u : x << 16);
                }
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bf16_t v = Vs[dt * 256 + i * 4];
                        if (finite16(v)) continue;
#pragma unroll
                        for (int t = 0; t < QT; ++t)
                            if (seen[t] >> slot & 1) O[t][dt][i] += w[t] * bf16_to_f(v);
                    }
            }
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            Op8 vo;
            vo.h[0] = *(const uint2 *)(VA + (dt * 64 + lane) * 4);
            vo.h[1] = *(const uint2 *)(VB + (dt * 64 + lane) * 4);
            if (odd) {   // what is not finite leaves the product
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!finite16(vo.w[e >> 1] >> ((e & 1) * 16))) vo.w[e >> 1] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
            }
#pragma unroll
            for (int t = 0; t < QT; ++t) O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo.v, pop[t].v, O[t][dt], 0, 0, 0);
        }
    };
    u32x4 rA[VEC], rB[VEC];   // two pairs in flight: the next one and the one after it
    int hA = 0, hB, h0, h1 = 0;
    hB = fetch(0, rB);
    if (n_pairs > 1) hA = fetch(1, rA);
    stash(0, rB, 0, hB);
    h0 = hB;
    __syncthreads();
    // iteration pp: registers hold pair pp + 1, pair pp + 2 is requested, pair pp is consumed from LDS
    for (int pp = 0; pp < n_pairs; pp += 2) {
        if (pp + 2 < n_pairs) hB = fetch(pp + 2, rB);
        compute(pp, 0, h0);
        if (pp + 1 < n_pairs) { stash(1, rA, pp + 1, hA); h1 = hA; }
        __syncthreads();
        if (pp + 1 >= n_pairs) break;
        if (pp + 3 < n_pairs) hA = fetch(pp + 3, rA);
        compute(pp + 1, 1, h1);
        if (pp + 2 < n_pairs) { stash(0, rB, pp + 2, hB); h0 = hB; }
        __syncthreads();
    }
    if (!active) return;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int qi = q0 + t * 16 + ln;
        float l = l_run[t];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (qi >= QR) continue;
        if (n_chunks == 1) {
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            bf16_t *op = (bf16_t *)a.t.t.out + (size_t)(s.first + qi / G) * a.t.t.out_stride + (hk * G + qi % G) * HD + lg * 4;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                const f32x4 o = O[t][dt] * inv;
                *(uint2 *)(op + dt * 16) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
            }
        } else {
            const size_t at = ((size_t)blockIdx.x * a.t.kv.n_kv_heads + hk) * QB + wave * 16 * QT + t * 16 + ln;
            float *op = a.part_o + at * HD + lg * 4;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(op + dt * 16) = O[t][dt];
            if (lg == 0) a.part_ml[at] = make_float2(m_run[t], l);
        }
    }
}

// The partial results of a block's items: out = sum_c 2^{c (m_c - M)} o_c / sum_c 2^{c (m_c - M)} l_c.  One workgroup 16 queries, 16 threads a query.
template <int HD, int QT>
__global__ __launch_bounds__(256) void tree_merge_k(MfmaArgs a)
{
    constexpr int QB = 64 * QT, V4 = HD / 4, PER = (V4 + 15) / 16;
    const int hk = blockIdx.y, G = a.G, part = blockIdx.x % (QB / 16), want = blockIdx.x / (QB / 16);
    const Place pl = place_of(a.t, G, QB, want, true);
    const int b = __builtin_amdgcn_readfirstlane(pl.b);
    if (b < 0) return;
    const Seq s = seq_of(a.t, b, G, QB);
    const int n_chunks = (s.tiles + pl.cp - 1) / pl.cp, block = want - pl.before;
    if (n_chunks == 1) return;   // written by the attention itself
    const int ql = part * 16 + (threadIdx.x >> 4), qi = block * QB + ql, x = threadIdx.x & 15;
    if (qi >= s.nodes * G) return;
    const size_t step = (size_t)s.blocks * a.t.kv.n_kv_heads * QB, at0 = ((size_t)(pl.item0 + block) * a.t.kv.n_kv_heads + hk) * QB + ql;
    float M = -INFINITY;
    for (int c = x; c < n_chunks; c += 16) M = fmaxf(M, a.part_ml[at0 + c * step].x);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    float L = 0.f;
    f32x4 o[PER] = {};
    for (int c = 0; c < n_chunks; ++c) {
        const float2 ml = a.part_ml[at0 + c * step];
        const float w = ml.x == -INFINITY ? 0.f : exp2f((ml.x - M) * a.c);
        L += ml.y * w;
        const f32x4 *src = (const f32x4 *)(a.part_o + (at0 + c * step) * HD);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (x + 16 * i < V4) o[i] += src[x + 16 * i] * w;
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    bf16_t *op = (bf16_t *)a.t.t.out + (size_t)(s.first + qi / G) * a.t.t.out_stride + (hk * G + qi % G) * HD;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (x + 16 * i < V4) *(uint2 *)(op + (x + 16 * i) * 4) = make_uint2(pack_bf16(o[i][0] * inv, o[i][1] * inv), pack_bf16(o[i][2] * inv, o[i][3] * inv));
}

// Queries of a wavefront in units of 16: by the most queries that a kv head has in a sequence.
int query_tiles(int queries) { return queries <= 64 ? 1 : 2; }

struct Shape { int qt; long blocks, items; };

Shape shape_of(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes)
{
    Shape s;
    const int queries = max_nodes * (n_q_heads / kv.n_kv_heads);
    s.qt = query_tiles(queries);
    s.blocks = (long)n_seqs * ((queries + 64 * s.qt - 1) / (64 * s.qt));
    s.items = s.blocks + (ITEMS + kv.n_kv_heads - 1) / kv.n_kv_heads;   // at most one shorter item a block besides ITEMS full ones
    return s;
}

template <int HD, int QT>
void mfma_go(hipStream_t s, const MfmaArgs &a, const Shape &sh, bool merge)
{
    hipLaunchKernelGGL((tree_mfma_k<HD, QT>), dim3(sh.items, a.t.kv.n_kv_heads), dim3(256), 0, s, a);
    if (merge) hipLaunchKernelGGL((tree_merge_k<HD, QT>), dim3(sh.blocks * 4 * QT, a.t.kv.n_kv_heads), dim3(256), 0, s, a);
}

template <int HD>
void mfma_t(hipStream_t s, const MfmaArgs &a, const Shape &sh, bool merge)
{
    if (sh.qt == 1) mfma_go<HD, 1>(s, a, sh, merge); else mfma_go<HD, 2>(s, a, sh, merge);
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

size_t tree_workspace_bytes(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes, int max_len)
{
    if (kv.dtype == 0) return 256;
    const Shape sh = shape_of(kv, n_q_heads, n_seqs, max_nodes);
    return (size_t)sh.items * kv.n_kv_heads * 64 * sh.qt * (kv.head_dim * 4 + 8) + 256;
}

void launch_tree_attention(hipStream_t s, const sdlm_kv &kv, int layer, const sdlm_tree_args &t, void *workspace, size_t workspace_bytes)
{
    TreeArgs a;
    a.kv = kv; a.t = t;
    a.pool = (const char *)kv.pool + (size_t)layer * kv.layer_stride * (kv.dtype == 0 ? 4 : 2);
    a.scale = 1.0f / sqrtf((float)kv.head_dim);
    if (kv.dtype == 0) { rows_t<float>(s, a); return; }
    MfmaArgs m;
    m.t = a;
    m.G = t.n_q_heads / kv.n_kv_heads;
    m.c = 1.4426950408889634f / sqrtf((float)kv.head_dim);
    const Shape sh = shape_of(kv, t.n_q_heads, t.n_seqs, t.max_nodes);
    m.part_o = (float *)workspace;
    m.part_ml = (float2 *)((char *)workspace + (size_t)sh.items * kv.n_kv_heads * 64 * sh.qt * kv.head_dim * 4);
    // One item a block whatever the lengths are: no merge.
    const long most = (t.max_nodes + 2 * PAGE - 2) / PAGE + kv.pages_per_seq;
    const bool merge = most > MIN_TILES;
    switch (kv.head_dim) {
    case 32: mfma_t<32>(s, m, sh, merge); break;
    case 64: mfma_t<64>(s, m, sh, merge); break;
    case 96: mfma_t<96>(s, m, sh, merge); break;
    default: mfma_t<128>(s, m, sh, merge); break;
    }
}

}  // namespace sdlm
