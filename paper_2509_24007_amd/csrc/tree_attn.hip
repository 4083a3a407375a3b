// Attention of drafted token trees over a K/V cache: every node of a sequence sees the sequence's first `length` positions, and of the nodes
// those that its mask names.
//   out[r, h] = sum_j p_j V[j], p = softmax over the seen keys of q[r, h] . K[j] / sqrt(d); a node that sees no key gets zeros.
#include <math.h>

#include <type_traits>

#include "ops.hpp"

namespace sdlm {

namespace {

struct TreeArgs {
    sdlm_kv kv;
    sdlm_tree_args t;
    const void *pool;   // this layer's tiles
    float scale;
};

// Small fp32 calls, one launch.  One workgroup a (node, query head).  The seen tiles, the prefix's and then the nodes', go four at a time to each of four wavefronts, which hold a running maximum, sum and output,
// merged at the end.  Scores: a key a lane, its features in pieces of 16 bytes.  Output: a feature a lane, four slots a load.  Bound by its chain of round trips (page, K, V) over as
// many trips as a wavefront has; every row reads the cache anew, so it is taken for few rows over short prefixes only, see few_rows (5 sequences of up to 300 positions and 40 nodes
// 13.7 us, with one wavefront a row 62).
template <int HD>
__global__ __launch_bounds__(256) void tree_rows_k(TreeArgs a)
{
    constexpr int FD = (HD + 63) / 64;
    const int r = blockIdx.x / a.t.n_q_heads, hq = blockIdx.x % a.t.n_q_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = a.t.n_q_heads / a.kv.n_kv_heads, hk = hq / G;
    int b = -1;   // the sequence whose nodes include r
    for (int i = lane; i < a.t.n_seqs; i += 64)
        if (r >= a.t.node_offsets[i] && r < a.t.node_offsets[i + 1]) b = i;
    for (int o = 32; o > 0; o >>= 1) b = max(b, __shfl_xor(b, o));
    b = __builtin_amdgcn_readfirstlane(b);
    if (b < 0) return;
    const int first = a.t.node_offsets[b], nodes = min(a.t.node_offsets[b + 1] - first, a.t.max_nodes);
    if (r - first >= nodes) return;
    const int len = min(max(a.kv.lengths[b], 0), a.kv.pages_per_seq * PAGE), base = a.t.node_base ? min(max(a.t.node_base[b], 0), a.t.node_pages * PAGE) : 0;
    const uint64_t *mask = (const uint64_t *)a.t.mask + (size_t)r * a.t.mask_words;
    const int n_prefix = (len + PAGE - 1) / PAGE, n_tiles = n_prefix + (base % PAGE + nodes + PAGE - 1) / PAGE;
    const size_t tile = (size_t)2 * PAGE * HD;
    const float *pool = (const float *)a.pool;
    __shared__ float q[HD];
    __shared__ __attribute__((aligned(16))) float ps[4][64];
    __shared__ float wm[4], wl[4], wo[4][HD];
    for (int i = threadIdx.x; i < HD; i += 256) q[i] = ((const float *)a.t.q)[(size_t)r * a.t.q_stride + hq * HD + i] * a.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[FD] = {};
    for (int t0 = wave * 4; t0 < n_tiles; t0 += 16) {
        const int t = t0 + (lane >> 4), slot = lane & 15;
        int page = -1;
        bool vis = false;
        if (t < n_prefix) {
            page = a.kv.page_table[(size_t)b * a.kv.pages_per_seq + t];
            vis = t * PAGE + slot < len;
        } else if (t < n_tiles) {
            const int u = t - n_prefix + base / PAGE, n = (t - n_prefix) * PAGE + slot - base % PAGE;
            if (u < a.t.node_pages) page = a.t.node_table[(size_t)b * a.t.node_pages + u];
            vis = n >= 0 && n < nodes && ((mask[n >> 6] >> (n & 63)) & 1);
        }
        vis = vis && page >= 0 && page < a.kv.n_tiles;
        float s = -INFINITY;
        if (vis) {
            const float *K = pool + ((size_t)page * a.kv.n_kv_heads + hk) * tile + slot * 8;
            float s4[4] = {};
#pragma unroll 4
            for (int i = 0; i < HD; i += 8) {
                const float4 x = *(const float4 *)(K + i * PAGE), y = *(const float4 *)(K + i * PAGE + 4);
                s4[0] += q[i] * x.x + q[i + 4] * y.x;
                s4[1] += q[i + 1] * x.y + q[i + 5] * y.y;
                s4[2] += q[i + 2] * x.z + q[i + 6] * y.z;
                s4[3] += q[i + 3] * x.w + q[i + 7] * y.w;
            }
            s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
        }
        float mx = s;
        for (int d = 32; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
        const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn;   // scores of -infinity weigh nothing, also where there are no others yet
        const float corr = m == -INFINITY ? 0.f : __expf(m - ref), p = vis ? __expf(s - ref) : 0.f;   // a NaN score stays one, whatever ref is
        m = mn;
        l = l * corr + p;
#pragma unroll
        for (int f = 0; f < FD; ++f) o[f] *= corr;
        ps[wave][lane] = p;   // read back by the same wavefront only
        __builtin_amdgcn_wave_barrier();
        const uint64_t seen = __ballot(vis);
        for (int tt = 0; tt < 4; ++tt) {
            const uint32_t sn = (uint32_t)(seen >> (tt * 16)) & 0xffffu;
            if (!sn) continue;
            const float *V = pool + ((size_t)__shfl(page, tt * 16) * a.kv.n_kv_heads + hk) * tile + PAGE * HD;
#pragma unroll
            for (int f = 0; f < FD; ++f) {
                const int i = lane + f * 64;
                if (i >= HD) continue;
#pragma unroll
                for (int sg = 0; sg < 4; ++sg) {
                    const float4 p4 = *(const float4 *)&ps[wave][tt * 16 + sg * 4], v = *(const float4 *)(V + v_off(sg * 4, i));
                    const float w[4] = {p4.x, p4.y, p4.z, p4.w}, x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[f] += sn >> (sg * 4 + e) & 1 ? w[e] * x[e] : 0.f;   // an unseen slot may hold anything
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
    if (lane == 0) { wm[wave] = m; wl[wave] = l; }
#pragma unroll
    for (int f = 0; f < FD; ++f)
        if (lane + f * 64 < HD) wo[wave][lane + f * 64] = o[f];
    __syncthreads();
    float M = -INFINITY, L = 0.f, w[4];
    for (int i = 0; i < 4; ++i) M = fmaxf(M, wm[i]);
    for (int i = 0; i < 4; ++i) { w[i] = wm[i] == -INFINITY ? (wl[i] != wl[i] ? wl[i] : 0.f) : __expf(wm[i] - M); L += wl[i] * w[i]; }
    for (int i = threadIdx.x; i < HD; i += 256) {
        float acc = 0.f;
        for (int k = 0; k < 4; ++k) acc += wo[k][i] * w[k];
        ((float *)a.t.out)[(size_t)r * a.t.out_stride + hq * HD + i] = L == 0.f ? 0.f : acc / L;
    }
}

// ------------------------------------------------------------------------------------------------ matrix-core path
// The queries of a sequence and kv head are its (node, query head) pairs, in blocks of 16 QT for each of four wavefronts; every tile that the workgroup
// brings to LDS serves the whole block.  A launch has as many workgroups as the chip holds at once, and the tiles of all blocks, one block behind the other, are
// dealt out to them in equal runs: no unit waits for another at the end, whatever the lengths are.  A workgroup's run may end inside a block; such a part leaves a
// maximum, a sum and an unnormalised output, and the parts of a block are merged by a second launch.  At most its first and its last part are incomplete, so a
// workgroup has two places for them.  fp32 tiles and operands take the instruction of 16 x 16 x 4, whose operands are neighbours in the tiles as they are.
// us, attention and merge, averages under the profiler (a call among others): 64 sequences of 2048 to 4096 positions, up to 16 nodes, 28 / 4 heads 112 + 11 (112: 413 MB, 3.7 TB/s);  4 of up to 8192, up to 256
// nodes, 16 / 2 heads 114 + 9 (103: 41 GFLOP, 400 TFLOP/s);  one of 512, 12 nodes 10 + 6 (16), a chain of round trips.  The wide trees' units are at the matrix instructions for 38 % of their time, at the vector
// instructions between the two products for 45 % and at LDS for 26 %, with two wavefronts a SIMD to overlap them.  The runs follow from the lengths by prefix sums over the sequences, a lane a sequence, that every wavefront makes for itself.
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
union Op8 { bf16x8 v; uint4 u; uint2 h[2]; uint32_t w[4]; };

constexpr int SLOTS = 512;            // workgroups that the chip holds at once, two a unit
constexpr int MIN_PAIRS = 2;          // fewest pairs of tiles a workgroup takes, where there are that many
constexpr float RESCALE_GAP = 8.0f;   // log2 units, see the running maximum below

__device__ inline bool finite16(uint32_t x) { return (x & 0x7f80u) != 0x7f80u; }   // of a bf16's bits
__device__ inline bool finite32(uint32_t x) { return (x & 0x7f800000u) != 0x7f800000u; }

__device__ inline void store4(float *p, const f32x4 &o) { *(f32x4 *)p = o; }
__device__ inline void store4(bf16_t *p, const f32x4 &o) { *(uint2 *)p = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])); }

struct MfmaArgs {
    TreeArgs t;
    float *part_o;      // [workgroup][first, last][query of the block][HD]
    float2 *part_ml;    // [workgroup][first, last][query of the block]: reference (log2), sum
    float c;            // log2(e) / sqrt(d)
    int G, groups;      // groups: workgroups for each kv head
};

struct Seq { int first, nodes, len, base, prefix_tiles, tiles, pairs, blocks; };

__device__ inline Seq seq_of(const TreeArgs &a, int b, int G, int qb)
{
    Seq s;
    s.first = min(max(a.t.node_offsets[b], 0), a.t.n_rows);
    s.nodes = min(max(min(a.t.node_offsets[b + 1], a.t.n_rows) - s.first, 0), a.t.max_nodes);
    s.len = min(max(a.kv.lengths[b], 0), a.kv.pages_per_seq * PAGE);
    s.base = a.t.node_base ? min(max(a.t.node_base[b], 0), a.t.node_pages * PAGE) : 0;
    s.prefix_tiles = (s.len + PAGE - 1) / PAGE;
    s.tiles = s.prefix_tiles + (s.base % PAGE + s.nodes + PAGE - 1) / PAGE;
    s.pairs = (s.tiles + 1) / 2;
    s.blocks = (s.nodes * G + qb - 1) / qb;
    return s;
}

// The same in every lane, and known to be: loops and branches over it stay scalar.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Exclusive prefix sums over 64 sequences, a lane a sequence, of their pairs of tiles (each block's) and of their blocks, and the sums.  The pairs of a launch fit 31 bits (checked on the host).
struct Sums { int pairs, blocks, all_pairs, all_blocks; };

__device__ inline Sums lane_sums(const TreeArgs &a, int b0, int G, int qb)
{
    const int lane = threadIdx.x & 63, n = min(a.t.n_seqs - b0, 64);
    int v = 0, w = 0;
    if (lane < n) { const Seq s = seq_of(a, b0 + lane, G, qb); w = s.blocks; v = w * s.pairs; }
    int x = v, y = w;
    for (int o = 1; o < n; o <<= 1) {
        const int u = __shfl_up(x, o), z = __shfl_up(y, o);
        if (lane >= o) { x += u; y += z; }
    }
    return Sums{x - v, y - w, __builtin_amdgcn_readlane(x, n - 1), __builtin_amdgcn_readlane(y, n - 1)};
}

// The run of workgroup w of a kv head: pairs w run .. (w + 1) run - 1.
__device__ inline int run_of(int all, int groups) { return max((all + groups - 1) / groups, MIN_PAIRS); }

__device__ inline int all_pairs(const TreeArgs &a, const Sums &first, int G, int qb)
{
    int sum = first.all_pairs;
    for (int b0 = 64; b0 < a.t.n_seqs; b0 += 64) sum += lane_sums(a, b0, G, qb).all_pairs;
    return sum;
}

// The sequence in which pair (or, by_block, block) `at` lies, and how many pairs and blocks are in front of it; b = -1: none.  first: the sums of the first 64 sequences.
struct Place { int b, blocks, pairs; };

__device__ inline Place place_of(const TreeArgs &a, const Sums &first, int G, int qb, int at, bool by_block)
{
    Sums m = first;
    int pairs = 0, blocks = 0;
    for (int b0 = 0; b0 < a.t.n_seqs; b0 += 64) {
        if (b0) m = lane_sums(a, b0, G, qb);
        if (at < (by_block ? blocks + m.all_blocks : pairs + m.all_pairs)) {   // the last lane whose first pair is not behind `at`: those without any share their first pair with the next
            const uint64_t not_behind = __ballot((by_block ? blocks + m.blocks : pairs + m.pairs) <= at && b0 + (int)(threadIdx.x & 63) < a.t.n_seqs);
            const int lane = 63 - __clzll((long long)not_behind);
            return Place{b0 + lane, blocks + __builtin_amdgcn_readlane(m.blocks, lane), pairs + __builtin_amdgcn_readlane(m.pairs, lane)};
        }
        pairs += m.all_pairs;
        blocks += m.all_blocks;
    }
    return Place{-1, 0, 0};
}

__device__ inline float max3(float a, float b, float c)   // of results of vector instructions; a NaN loses
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

template <typename T, int HD, int QT>
__global__ __launch_bounds__(256, 2) void tree_mfma_k(MfmaArgs a)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int E = 16 / sizeof(T);                                                              // elements in 16 bytes
    constexpr int QB = 64 * QT, NK = HD / 32, ND = HD / 16, TILE = 2 * PAGE * HD, VEC = HD / (4 * E);   // VEC: 16-byte loads of a thread for a pair of tiles
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), ln = lane & 15, lg = lane >> 4, G = a.G;
    // Workgroups are dealt to the eight dies in turn: each die gets a stretch of neighbouring runs, whose blocks read the same tiles.
    const int per_die = (gridDim.x + 7) / 8, id = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3), hk = id / a.groups;
    if (hk >= a.t.kv.n_kv_heads) return;
    const Sums sums = lane_sums(a.t, 0, G, QB);
    const int all = all_pairs(a.t, sums, G, QB), run = run_of(all, a.groups);
    const int end = (int)min((long)all, (long)(id % a.groups + 1) * run);
    int from = (int)min((long)all, (long)(id % a.groups) * run);
    __shared__ __attribute__((aligned(16))) T kv[2][2 * TILE];   // two pairs of tiles, each as in the pool
    __shared__ int strange[2][4];   // per wavefront: whether its part of the pair's values has some that are not finite (not for pairs that every query sees whole)
    const T *pool = (const T *)a.t.pool;
    for (int part = 0; from < end; ++part) {
    const Place pl = place_of(a.t, sums, G, QB, from, false);
    const int b = uniform(pl.b);
    if (b < 0) return;
    const Seq s = seq_of(a.t, b, G, QB);
    const int inside = from - uniform(pl.pairs), block = inside / s.pairs, p0 = inside % s.pairs;
    const int n_pairs = min(s.pairs - p0, end - from), u0 = 2 * p0, u1 = min(s.tiles, u0 + 2 * n_pairs);
    const bool complete = n_pairs == s.pairs;
    from += n_pairs;
    const int q0 = block * QB + wave * 16 * QT, QR = s.nodes * G;
    const bool active = q0 < QR;
    const int32_t *ptab = a.t.kv.page_table + (size_t)b * a.t.kv.pages_per_seq, *ntab = a.t.t.node_table + (size_t)b * a.t.t.node_pages;
    const int node_tile0 = s.base / PAGE - s.prefix_tiles, shift0 = s.prefix_tiles * PAGE + s.base % PAGE;   // tile u >= prefix_tiles: entry u + node_tile0; its slot i is node u 16 + i - shift0

    // This wavefront's queries, B operands: lane (query ln, group lg) holds features 32 kk + 8 lg .. + 7 of step kk; fp32: features 8 o + 2 lg and the next, a step each.
    Op8 qop[QT][F32 ? 1 : NK];
    float qf[QT][F32 ? HD / 4 : 1];
    int mrow[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int qi = q0 + t * 16 + ln;
        const bool ok = qi < QR;
        const int row = s.first + (ok ? qi / G : 0), h = hk * G + (ok ? qi % G : 0);
        const T *qp = (const T *)a.t.t.q + (size_t)row * a.t.t.q_stride + h * HD + lg * (F32 ? 2 : 8);
        mrow[t] = row;
        if constexpr (F32) {
#pragma unroll
            for (int o = 0; o < HD / 8; ++o) {
                float2 x = make_float2(0.f, 0.f);
                if (ok) x = *(const float2 *)(qp + o * 8);
                qf[t][2 * o] = x.x;
                qf[t][2 * o + 1] = x.y;
            }
        } else {
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                qop[t][kk].u = make_uint4(0, 0, 0, 0);
                if (ok) qop[t][kk].u = *(const uint4 *)(qp + kk * 32);
            }
        }
    }
    f32x4 O[QT][ND];
    float m_run[QT], l_run[QT];

    // Pages of 64 tiles, one a lane, and of the next 64: a lookup of its own in front of every pair would put a memory round trip into every iteration.  -1: there is none.
    auto pages = [&](int w) -> int {
        const int u = u0 + w * 64 + lane;
        int p = -1;
        if (u < s.prefix_tiles) { if (u < u1) p = ptab[u]; }
        else if (u < u1 && u + node_tile0 < a.t.t.node_pages) p = ntab[u + node_tile0];
        return p < a.t.kv.n_tiles ? p : -1;
    };
    int pg, pg_next;
    bool careful = false;   // the second try of a part whose values are not all finite, see its end
    // a pair in flight: its tiles' contents, and whether they exist.  Called for pairs in ascending order.
    auto fetch = [&](int pp, u32x4 (&r)[VEC]) -> int {
        if ((pp & 31) == 0 && pp > 0) {
            pg = pg_next;
            if (pp + 32 < n_pairs) pg_next = pages(pp / 32 + 1);
        }
        const int pA = __builtin_amdgcn_readlane(pg, 2 * (pp & 31)), pB = __builtin_amdgcn_readlane(pg, 2 * (pp & 31) + 1);
        const T *tA = pool + ((size_t)max(pA, 0) * a.t.kv.n_kv_heads + hk) * TILE, *tB = pool + ((size_t)max(pB >= 0 ? pB : pA, 0) * a.t.kv.n_kv_heads + hk) * TILE;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const T *t = wave * 64 + 256 * i < TILE / E ? tA : tB - TILE;   // a wavefront's part lies in one tile
            r[i] = *(const u32x4 *)(t + (unsigned)(tid + 256 * i) * E);
        }
        return (pA >= 0 ? 1 : 0) | (pB >= 0 ? 2 : 0);
    };
    auto is_whole = [&](int pp, int have) { return !careful && have == 3 && (u0 + 2 * pp + 2) * PAGE <= s.len; };   // every key of the pair is seen by every query
    auto stash = [&](int buf, const u32x4 (&r)[VEC], int pp, int have) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) *(u32x4 *)(&kv[buf][0] + (size_t)(tid + 256 * i) * E) = r[i];
        if (is_whole(pp, have)) return;
        bool any = false;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if ((tid + 256 * i) % (TILE / E) >= TILE / E / 2)
#pragma unroll
                for (int k = 0; k < 4; ++k) any |= F32 ? !finite32(r[i][k]) : !finite16(r[i][k]) || !finite16(r[i][k] >> 16);
        any = __any(any);
        if (lane == 0) strange[buf][wave] = any;
    };
    auto compute = [&](int pp, int buf, int have) {
        if (!active) return;
        const int uA = u0 + 2 * pp;
        const T *KA = &kv[buf][0], *KB = KA + TILE;
        f32x4 sA[QT], sB[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) { sA[t] = f32x4{0.f, 0.f, 0.f, 0.f}; sB[t] = sA[t]; }
        const T *VA = KA + PAGE * HD, *VB = KB + PAGE * HD;
        Op8 vo[F32 ? 1 : ND];
        if constexpr (F32) {
            // keys as rows, features 8 o + {0, 2, 4, 6} and 8 o + {1, 3, 5, 7} as the four columns of a step: a lane's two are neighbours
#pragma unroll
            for (int o = 0; o < HD / 8; ++o) {
                const float2 ka = *(const float2 *)(KA + o * 128 + ln * 8 + lg * 2), kb = *(const float2 *)(KB + o * 128 + ln * 8 + lg * 2);
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    sA[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.x, qf[t][2 * o], sA[t], 0, 0, 0);
                    sB[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kb.x, qf[t][2 * o], sB[t], 0, 0, 0);
                    sA[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.y, qf[t][2 * o + 1], sA[t], 0, 0, 0);
                    sB[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kb.y, qf[t][2 * o + 1], sB[t], 0, 0, 0);
                }
            }
        } else {
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
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {   // requested here, used behind the softmax
                vo[dt].h[0] = *(const uint2 *)(VA + (dt * 64 + lane) * 4);
                vo[dt].h[1] = *(const uint2 *)(VB + (dt * 64 + lane) * 4);
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
        // Exponents of 2, against a reference that is a maximum of earlier scores: x = c s - ref.  It only moves when it is exceeded by more than RESCALE_GAP (2^x stays
        // below 2^RESCALE_GAP, harmless in fp32 sums and bf16 products); only then is the maximum taken over the query's four lanes and are the accumulators rescaled.
        float x[QT][8], mx[QT];
        bool grows = false;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float ref = m_run[t] == -INFINITY ? 0.f : m_run[t];
#pragma unroll
            for (int v = 0; v < 4; ++v) { x[t][v] = fmaf(sA[t][v], a.c, -ref); x[t][4 + v] = fmaf(sB[t][v], a.c, -ref); }
            mx[t] = max3(max3(x[t][0], x[t][1], x[t][2]), max3(x[t][3], x[t][4], x[t][5]), max3(x[t][6], x[t][7], x[t][7]));
            grows |= mx[t] > (m_run[t] == -INFINITY ? -INFINITY : RESCALE_GAP);
        }
        if (__any(grows)) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const float ref = m_run[t] == -INFINITY ? 0.f : m_run[t];
                mx[t] = fmaxf(mx[t], __shfl_xor(mx[t], 16));
                mx[t] = fmaxf(mx[t], __shfl_xor(mx[t], 32));
                const float m_new = fmaxf(m_run[t], mx[t] + ref);
                const float to = m_new == -INFINITY ? 0.f : m_new, corr = m_run[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[t] - to);   // without a reference nothing has been added
                l_run[t] *= corr;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) O[t][dt] *= corr;
                m_run[t] = m_new;
#pragma unroll
                for (int v = 0; v < 4; ++v) { x[t][v] = fmaf(sA[t][v], a.c, -to); x[t][4 + v] = fmaf(sB[t][v], a.c, -to); }
            }
        }
        // bf16: a weight goes into the product as two operands, its rounding to bf16 and what that leaves, so that it keeps 2^-16 of itself.  One rounding alone is up to 2^-8 of each weight, as much
        // again as the output's own (relative error against 64 bits, and us a call for 64 sequences and for 4 wide trees as above: one operand 2.3e-3, 107 and 91; two 1.66e-3, which is the
        // output's rounding alone, 113 and 109).
        Op8 pop[QT], rest[QT];
        f32x4 pA[QT], pB[QT];   // the weights of the slots 4 lg + v of each tile
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                pA[t][v] = __builtin_amdgcn_exp2f(x[t][v]);
                pB[t][v] = __builtin_amdgcn_exp2f(x[t][4 + v]);
            }
            l_run[t] += (pA[t][0] + pA[t][1]) + (pA[t][2] + pA[t][3]) + (pB[t][0] + pB[t][1]) + (pB[t][2] + pB[t][3]);
            if constexpr (!F32)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x0 = i < 2 ? pA[t][2 * i] : pB[t][2 * i - 4], x1 = i < 2 ? pA[t][2 * i + 1] : pB[t][2 * i - 3];
                    const uint32_t w = pack_bf16(x0, x1);
                    pop[t].w[i] = w;
                    rest[t].w[i] = pack_bf16(x0 - __uint_as_float(w << 16), x1 - __uint_as_float(w & 0xffff0000u));
                }
        }
        // A slot that a query does not see may hold anything, and 0 times a value that is not finite is not 0.  Such values are added one by one for the queries that see them.
        const bool odd = !whole && (strange[buf][0] | strange[buf][1] | strange[buf][2] | strange[buf][3]);
        if (odd) {
#pragma unroll 1
            for (int slot = 0; slot < 32; ++slot) {
                const int from = (slot >> 2 & 3) * 16 + ln;   // the lane that has the query's weight for this slot
                const T *Vs = (slot < 16 ? VA : VB) + ((slot >> 2 & 3) * 16 + lg * 4) * 4 + (slot & 3);
                float w[QT];
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    const int k = slot & 3;
                    const f32x4 mine = slot < 16 ? pA[t] : pB[t];
                    const float lo = k & 1 ? mine[1] : mine[0], hi = k & 1 ? mine[3] : mine[2];
                    w[t] = __shfl(k & 2 ? hi : lo, from);
                }
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = to_f<T>(Vs[dt * 256 + i * 4]);
                        if (finite32(__float_as_uint(v))) continue;
#pragma unroll
                        for (int t = 0; t < QT; ++t)
                            if (seen[t] >> slot & 1) O[t][dt][i] += w[t] * v;
                    }
            }
            if constexpr (!F32) {
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!finite16(vo[dt].w[e >> 1] >> ((e & 1) * 16))) vo[dt].w[e >> 1] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
            }
        }
        if constexpr (F32) {
            // a lane's four values are the slots 4 lg + v of feature dt 16 + ln, its weights those of the same slots: a step for each v
            auto values = [&](auto clean) {
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    f32x4 va = *(const f32x4 *)(VA + (dt * 64 + lane) * 4), vb = *(const f32x4 *)(VB + (dt * 64 + lane) * 4);
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        if constexpr (clean) {
                            if (!finite32(__float_as_uint(va[v]))) va[v] = 0.f;
                            if (!finite32(__float_as_uint(vb[v]))) vb[v] = 0.f;
                        }
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
                            O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(va[v], pA[t][v], O[t][dt], 0, 0, 0);
                            O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vb[v], pB[t][v], O[t][dt], 0, 0, 0);
                        }
                    }
                }
            };
            if (odd) values(std::true_type{}); else values(std::false_type{});
        } else {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo[dt].v, pop[t].v, O[t][dt], 0, 0, 0);
                    O[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo[dt].v, rest[t].v, O[t][dt], 0, 0, 0);
                }
        }
    };
    for (;;) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m_run[t] = -INFINITY; l_run[t] = 0.f;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) O[t][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    pg = pages(0);
    pg_next = n_pairs > 32 ? pages(1) : -1;
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
    if constexpr (F32) break;
    else {
        // An infinite value times the two operands of a weight is infinity less infinity, or times nothing.  Where a result is not finite, the part is computed once more with such values taken out
        // of every tile and added with the whole weight.
        bool odd = false;
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) odd |= !finite32(__float_as_uint(O[t][dt][i]));
        if (careful || !__syncthreads_or(odd)) break;
        careful = true;
    }
    }
    if (active) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int qi = q0 + t * 16 + ln;
            float l = l_run[t];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (qi >= QR) continue;
            if (complete) {
                const float inv = l == 0.f ? 0.f : 1.0f / l;
                T *op = (T *)a.t.t.out + (size_t)(s.first + qi / G) * a.t.t.out_stride + (hk * G + qi % G) * HD + lg * 4;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) store4(op + dt * 16, O[t][dt] * inv);
            } else {
                const size_t at = ((size_t)id * 2 + (part > 0)) * QB + wave * 16 * QT + t * 16 + ln;
                float *op = a.part_o + at * HD + lg * 4;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(op + dt * 16) = O[t][dt];
                if (lg == 0) a.part_ml[at] = make_float2(m_run[t], l);
            }
        }
    }
    }
}

// The parts of a block: out = sum_c 2^{m_c - M} o_c / sum_c 2^{m_c - M} l_c.  One workgroup 16 queries, 16 threads a query.
template <typename T, int HD, int QT>
__global__ __launch_bounds__(256) void tree_merge_k(MfmaArgs a)
{
    constexpr int QB = 64 * QT, V4 = HD / 4, PER = (V4 + 15) / 16;
    const int hk = blockIdx.y, G = a.G, part = blockIdx.x % (QB / 16), want = blockIdx.x / (QB / 16);
    const Sums sums = lane_sums(a.t, 0, G, QB);
    const int run = run_of(all_pairs(a.t, sums, G, QB), a.groups);
    const Place pl = place_of(a.t, sums, G, QB, want, true);
    const int b = uniform(pl.b);
    if (b < 0) return;
    const Seq s = seq_of(a.t, b, G, QB);
    const int block = want - pl.blocks;
    const int x0 = pl.pairs + block * s.pairs, w0 = x0 / run, n_parts = (x0 + s.pairs - 1) / run - w0 + 1;
    if (n_parts == 1) return;   // written by the attention itself
    const int ql = part * 16 + (threadIdx.x >> 4), qi = block * QB + ql, x = threadIdx.x & 15;
    if (qi >= s.nodes * G) return;
    const int late = w0 * run < x0;   // the first workgroup's run began in front of this block: the part is its last one
    const size_t id0 = (size_t)hk * a.groups + w0;
    auto at = [&](int c) { return ((id0 + c) * 2 + (c == 0 ? late : 0)) * QB + ql; };
    float M = -INFINITY;
    for (int c = x; c < n_parts; c += 16) M = fmaxf(M, a.part_ml[at(c)].x);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    float L = 0.f;
    f32x4 o[PER] = {};
    for (int c = 0; c < n_parts; ++c) {
        const float2 ml = a.part_ml[at(c)];
        const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
        L += ml.y * w;
        const f32x4 *src = (const f32x4 *)(a.part_o + at(c) * HD);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (x + 16 * i < V4) o[i] += src[x + 16 * i] * w;
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    T *op = (T *)a.t.t.out + (size_t)(s.first + qi / G) * a.t.t.out_stride + (hk * G + qi % G) * HD;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (x + 16 * i < V4) store4(op + (x + 16 * i) * 4, o[i] * inv);
}

// Queries of a wavefront in units of 16: by the most queries that a kv head has in a sequence.  One for up to 64, so that all four wavefronts have some; beyond, two, which reads
// every tile half as often from memory and LDS.  us, one / two: 64 sequences of 3000 positions, 7 queries 84 / 88, 56 queries 98 / 105, 70 queries 113 / 111, 112 queries 126 / 124;  4 trees of 1200 to
// 2048 queries over 6144 positions 120 / 103.  Three would need more registers than two workgroups a unit leave.
int query_tiles(int queries) { return queries <= 64 ? 1 : 2; }

// fp32 calls that one launch of tree_rows_k serves faster: by the length of the longest prefix as the caller names it or what the table holds (a wrong one costs time, nothing else), and the
// keys that all rows read together.  us, rows / matrix cores: 1 sequence of 300 positions, 8 nodes, 4 heads 14.2 / 16.8;  500 positions, 12 nodes, 12 heads 14.6 / 20.7;  3 of 700, 30 nodes,
// 6 heads 14.2 / 19.9;  beyond: 1 of 4000, 12 nodes, 12 heads 71.7 / 42.9;  4 of 1000, 16 nodes, 28 heads 84.4 / 34.5;  4 of 4000, 128 nodes, 40 heads 8305 / 386 (109 TFLOP/s of the 154 that a library's fp32 product reaches here).
bool few_rows(const sdlm_kv &kv, const sdlm_tree_args &t)
{
    const double len = t.max_len ? t.max_len : (double)kv.pages_per_seq * PAGE;
    return kv.dtype == 0 && len <= 1024 && (double)t.n_rows * t.n_q_heads * (len + t.max_nodes) <= 512.0 * 1024;
}

struct Shape { int qt, groups; long blocks; };

Shape shape_of(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes)
{
    Shape s;
    const int queries = max_nodes * (n_q_heads / kv.n_kv_heads);
    s.qt = kv.dtype == 0 ? 1 : query_tiles(queries);   // fp32: tiles of twice the bytes
    s.blocks = (long)n_seqs * ((queries + 64 * s.qt - 1) / (64 * s.qt));
    s.groups = kv.n_kv_heads >= SLOTS ? 1 : SLOTS / kv.n_kv_heads;
    return s;
}

// The places for the parts of one workgroup of each kv head.
size_t run_bytes(int n_kv_heads, int head_dim, int qt) { return (size_t)n_kv_heads * 2 * 64 * qt * (head_dim * 4 + 8); }

template <typename T, int HD, int QT>
void mfma_go(hipStream_t s, const MfmaArgs &a, const Shape &sh)
{
    const unsigned n = (unsigned)(sh.groups * a.t.kv.n_kv_heads + 7) / 8 * 8;
    hipLaunchKernelGGL((tree_mfma_k<T, HD, QT>), dim3(n), dim3(256), 0, s, a);
    hipLaunchKernelGGL((tree_merge_k<T, HD, QT>), dim3(sh.blocks * 4 * QT, a.t.kv.n_kv_heads), dim3(256), 0, s, a);
}

template <int HD>
void mfma_t(hipStream_t s, const MfmaArgs &a, const Shape &sh)
{
    if (a.t.kv.dtype == 0) mfma_go<float, HD, 1>(s, a, sh);
    else if (sh.qt == 1) mfma_go<bf16_t, HD, 1>(s, a, sh);
    else mfma_go<bf16_t, HD, 2>(s, a, sh);
}

void rows(hipStream_t s, const TreeArgs &a)
{
    const dim3 grid((unsigned)a.t.n_rows * a.t.n_q_heads), block(256);
    switch (a.kv.head_dim) {
    case 32: hipLaunchKernelGGL(tree_rows_k<32>, grid, block, 0, s, a); break;
    case 64: hipLaunchKernelGGL(tree_rows_k<64>, grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL(tree_rows_k<96>, grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL(tree_rows_k<128>, grid, block, 0, s, a); break;
    }
}

}  // namespace

bool tree_fits(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes)
{
    const long pairs = (kv.pages_per_seq + (max_nodes + 2 * PAGE - 2) / PAGE + 1) / 2, blocks = ((long)max_nodes * (n_q_heads / kv.n_kv_heads) + 63) / 64;
    return (double)n_seqs * blocks * pairs < 2147000000.0 && (double)n_seqs * blocks < (double)(1 << 21);   // the second launch: 4 or 8 workgroups of 256 threads a block
}

size_t tree_workspace_bytes(const sdlm_kv &kv, int n_q_heads, int n_seqs, int max_nodes, int max_len)
{
    const Shape sh = shape_of(kv, n_q_heads, n_seqs, max_nodes);
    return sh.groups * run_bytes(kv.n_kv_heads, kv.head_dim, sh.qt) + 256;
}

size_t tree_workspace_least(int n_kv_heads, int head_dim, int dtype) { return run_bytes(n_kv_heads, head_dim, dtype == 0 ? 1 : 2) + 256; }

void launch_tree_attention(hipStream_t s, const sdlm_kv &kv, int layer, const sdlm_tree_args &t, void *workspace, size_t workspace_bytes)
{
    TreeArgs a;
    a.kv = kv; a.t = t;
    a.pool = (const char *)kv.pool + (size_t)layer * kv.layer_stride * (kv.dtype == 0 ? 4 : 2);
    a.scale = 1.0f / sqrtf((float)kv.head_dim);
    if (few_rows(kv, t)) { rows(s, a); return; }
    MfmaArgs m;
    m.t = a;
    m.G = t.n_q_heads / kv.n_kv_heads;
    m.c = 1.4426950408889634f / sqrtf((float)kv.head_dim);
    Shape sh = shape_of(kv, t.n_q_heads, t.n_seqs, t.max_nodes);
    // A context lends less workspace than a caller has to: fewer, longer runs.
    const size_t fit = (workspace_bytes - 256) / run_bytes(kv.n_kv_heads, kv.head_dim, sh.qt);   // at least 1: tree_workspace_least
    if (fit < (size_t)sh.groups) sh.groups = (int)fit;
    m.part_o = (float *)workspace;
    m.part_ml = (float2 *)((char *)workspace + (size_t)sh.groups * kv.n_kv_heads * 2 * 64 * sh.qt * kv.head_dim * 4);
    m.groups = sh.groups;
    switch (kv.head_dim) {
    case 32: mfma_t<32>(s, m, sh); break;
    case 64: mfma_t<64>(s, m, sh); break;
    case 96: mfma_t<96>(s, m, sh); break;
    default: mfma_t<128>(s, m, sh); break;
    }
}

}  // namespace sdlm
