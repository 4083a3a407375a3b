// Drawing tokens from logits: temperature, top-k, top-p, min-p and a given uniform number, row by row.
//
// The tokens of a row are ordered by logit, equal ones by index.  All filters keep a first part of that order, and the uniform number
// picks from the kept part in that order, so the kernel never sorts: each step looks for the first token whose running count or
// running weight passes a bound, by digits of the order-preserving integer of the logit.
// Weights w = e^((z - max) / t) are integers in units of 2^-44 of the largest: their sums do not depend on the order of the threads,
// and their error (2^-45 a token) is far below the weight of any token that a draw could fall on.
#include "ops.hpp"

namespace sdlm {

namespace {

constexpr int TH = 1024;
typedef unsigned long long u64;
constexpr double ONE = 17592186044416.0;   // 2^44

__device__ inline float canon(float z)   // NaN is never drawn; the two zeros are equal
{
    return z != z ? -INFINITY : z == 0.f ? 0.f : z;
}
__device__ inline uint32_t key_of(float z)
{
    const uint32_t b = __float_as_uint(z);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ inline float of_key(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

template <typename T>
struct Row {
    const T *z;
    int V;
    __device__ float at(int i) const { return canon(to_f<T>(z[i])); }
};

struct Weigh {
    double M, c;   // largest logit, log2(e) / t
    __device__ u64 operator()(float z) const
    {
        if ((double)z == M) return (u64)ONE;   // also where the largest is infinite
        const double y = ((double)z - M) * c;
        return y < -46.0 ? 0ull : (u64)(exp2(y) * ONE + 0.5);
    }
};

// What a search found: the token's key, how many of the tokens with that key come up to it (1: the first), count and weight of the order up to and including it.
struct Found { uint32_t key; int rank; u64 mass; };

struct Shared {
    u64 mass[256];
    uint32_t cnt[256];
    u64 red[TH / 64];
    Found f;
    uint32_t prefix;
    u64 acc_mass, acc_cnt;
    int hit;
};

template <typename F>
__device__ inline u64 block_reduce(Shared &sh, u64 v, F f)
{
    for (int o = 32; o > 0; o >>= 1) v = f(v, (u64)__shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh.red[0];
    for (int i = 1; i < TH / 64; ++i) v = f(v, sh.red[i]);
    return v;
}

enum { BY_COUNT, MASS_AT_LEAST, MASS_ABOVE };

// The first token whose running count (weight) is at least, or above, `bound`.  The caller makes sure that there is one among the tokens above -infinity.
template <typename T>
__device__ Found search(Shared &sh, const Row<T> &row, const Weigh &w, int by, u64 bound)
{
    const int tid = threadIdx.x;
    if (tid == 0) { sh.prefix = 0; sh.acc_mass = 0; sh.acc_cnt = 0; }
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) { sh.mass[tid] = 0; sh.cnt[tid] = 0; }
        __syncthreads();
        const uint32_t prefix = sh.prefix;
        for (int i = tid; i < row.V; i += TH) {
            const float z = row.at(i);
            const uint32_t k = key_of(z);
            if (z == -INFINITY || (shift < 24 && (k >> (shift + 8)) != prefix)) continue;
            atomicAdd(&sh.cnt[(k >> shift) & 255], 1u);
            atomicAdd(&sh.mass[(k >> shift) & 255], w(z));
        }
        __syncthreads();
        if (tid == 0) {
            u64 m = sh.acc_mass, n = sh.acc_cnt;
            int last = -1, d = 255;
            for (; d >= 0; --d) {
                if (!sh.cnt[d]) continue;
                last = d;
                const u64 m1 = m + sh.mass[d], n1 = n + sh.cnt[d];
                if (by == BY_COUNT ? n1 >= bound : by == MASS_AT_LEAST ? m1 >= bound : m1 > bound) break;
                m = m1; n = n1;
            }
            if (d < 0) { d = last < 0 ? 0 : last; m -= sh.mass[d]; n -= sh.cnt[d]; }   // not passed: the last token
            sh.prefix = prefix << 8 | d;
            sh.acc_mass = m; sh.acc_cnt = n;
        }
        __syncthreads();
    }
    if (tid == 0) {
        const uint32_t ties = sh.cnt[sh.prefix & 255];
        const u64 each = w(of_key(sh.prefix)), m = sh.acc_mass;
        u64 r = ties;
        if (by == BY_COUNT) r = bound - sh.acc_cnt;
        else if (each) { const u64 lack = by == MASS_AT_LEAST ? bound - m : bound - m + 1; r = (lack + each - 1) / each; }
        if ((by != BY_COUNT && bound < m) || r < 1) r = 1;
        if (r > ties) r = ties;
        sh.f.key = sh.prefix; sh.f.rank = (int)r; sh.f.mass = m + r * each;
    }
    __syncthreads();
    const Found f = sh.f;
    __syncthreads();
    return f;
}

// Index of the rank-th token with this key.
template <typename T>
__device__ int index_of(Shared &sh, const Row<T> &row, uint32_t key, int rank)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    if (threadIdx.x == 0) sh.hit = -1;
    for (int i0 = 0; i0 < row.V; i0 += TH) {
        const int i = i0 + threadIdx.x;
        const bool eq = i < row.V && key_of(row.at(i)) == key;
        const u64 bal = __ballot(eq);
        __syncthreads();
        if (lane == 0) sh.red[wave] = __popcll(bal);
        __syncthreads();
        int at = before;
        for (int q = 0; q < TH / 64; ++q) { if (q < wave) at += (int)sh.red[q]; before += (int)sh.red[q]; }
        if (eq && at + __popcll(bal & ((1ull << lane) - 1)) == rank - 1) sh.hit = i;
        if (before >= rank) break;
    }
    __syncthreads();
    return sh.hit;
}

template <typename T>
__global__ __launch_bounds__(TH) void sample_k(sdlm_sample_args a)
{
    __shared__ Shared sh;
    const int r = blockIdx.x;
    const Row<T> row{(const T *)a.logits + (size_t)r * a.row_stride, a.vocab};
    uint32_t kmax = 0;
    for (int i = threadIdx.x; i < row.V; i += TH) kmax = max(kmax, key_of(row.at(i)));
    kmax = (uint32_t)block_reduce(sh, kmax, [](u64 x, u64 y) { return x > y ? x : y; });
    const float M = of_key(kmax), t = a.temperature ? a.temperature[r] : 1.f;
    int id = -1;
    float prob = 0.f;
    if (M == -INFINITY) {
        // every token is masked
    } else if (!(t > 0.f)) {
        id = index_of(sh, row, kmax, 1);
        prob = 1.f;
    } else {
        const Weigh w{(double)M, 1.4426950408889634 / (double)t};
        const int k = a.top_k ? a.top_k[r] : 0;
        const float p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f;
        auto add = [](u64 x, u64 y) { return x + y; };
        u64 n = 0, m = 0, mm = 0;
        const double least = fmin((double)mp, 1.0) * ONE;
        for (int i = threadIdx.x; i < row.V; i += TH) {
            const float z = row.at(i);
            const u64 x = z == -INFINITY ? 0 : w(z);
            n += z > -INFINITY; m += x;
            mm += (double)x >= least ? x : 0;
        }
        n = block_reduce(sh, n, add); m = block_reduce(sh, m, add); mm = block_reduce(sh, mm, add);
        u64 kept = m;
        if (k > 0 && (u64)k < n) kept = search(sh, row, w, BY_COUNT, (u64)k).mass;
        if (p < 1.f) kept = search(sh, row, w, MASS_AT_LEAST, (u64)ceil(fmax((double)p, 0.0) * (double)kept)).mass;
        if (mp > 0.f && mm < kept) kept = mm;
        const float u = a.u[r];
        const u64 at = (u64)(fmin(fmax((double)u, 0.0), 1.0) * (double)kept);
        const Found f = search(sh, row, w, MASS_ABOVE, min(at, kept - 1));
        id = index_of(sh, row, f.key, f.rank);
        prob = (float)((double)w(of_key(f.key)) / (double)kept);
    }
    if (threadIdx.x == 0) {
        a.ids[r] = id;
        if (a.prob) a.prob[r] = prob;
    }
}

}  // namespace

size_t sample_workspace_bytes(int rows, int vocab) { return 256; }

void launch_sample(hipStream_t s, const sdlm_sample_args &a, void *workspace)
{
    if (a.dtype == 0) hipLaunchKernelGGL(sample_k<float>, dim3(a.rows), dim3(TH), 0, s, a);
    else hipLaunchKernelGGL(sample_k<bf16_t>, dim3(a.rows), dim3(TH), 0, s, a);
}

}  // namespace sdlm
