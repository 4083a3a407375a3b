// Drawing tokens from logits: temperature, top-k, top-p, min-p and a given uniform number, row by row.
//
// The tokens of a row are ordered by logit, equal ones by index.  All filters keep a first part of that order, and the uniform number picks from the kept part
// in that order.  Weights are integers in units of 2^-44 of the largest (or of the power of two above it): their sums do not depend on the order of the threads, and
// their error (2^-45 of the largest a token; 2^-44 of it and 2^-29 of itself where the histogram counts) is far below the weight of any token that a draw could fall on.
//
// Two launches.  The first reads the logits once, all units together: a thread takes 64 of them and leaves the maxima of its runs, and for a row whose filters need the
// weight of the whole row (no top-k) a workgroup also leaves a histogram of the weights over 1/32 octaves.  The second has a workgroup a row, which sorts only what matters:
//   - top-k: the k-th largest of the runs' maxima is no more than the k-th largest logit, so the candidates are what reaches it, in the few runs that do;
//   - min-p: the candidates are what reaches min_p of the largest;
//   - otherwise the histogram says in which bin the weight passes top_p, and in which bin the draw falls, and the candidates are that bin.
// Where a row has too few runs for its top-k, the k-th logit itself is searched by digits.  Where more than CAND candidates come together, or where the exponents leave the histogram's range, the row is searched by digits
// of the logits' order-preserving integers instead, without sorting, in a dozen passes.  Those are: top-k beyond CAND; thousands of equal logits; a min-p that more than CAND tokens reach; and without top-k
// or min-p rows so flat that a bin, which is 0.0217 t wide in logits, holds more than CAND: one of V logits that fall off as e^(-z / s) does where 0.0217 V t / s is above CAND (152064 and s = 1.1: t = 1.4), and with an
// infinite temperature any with more than CAND logits.
//
// us: one row of 151936 fp32 5 + 13, 256 rows of 152064 with mixed settings 52 + 46, 33 rows of 33003 bf16 13 + 28.  The first launch is bound by the read where no row asks for weights (256 rows 39, 4.0 TB/s),
// else by the weights' instructions.  The second is a chain of scans and synchronisations in one workgroup, whose longest part, where a bound lies far down a flat tail, is the read of the whole row (about
// 25 each time, by its instructions).  256 rows with top_k = 2048 76, 4000 (the k-th by digits) 340, 5000 (all by digits) 732; 36 rows of 7452 bf16 with
// top_k = 1000, which have fewer runs than that, 66 (by digits 108).  Flat rows (256 of 152064, s = 1.1) with top-p 0.99: t = 1.3 159, from 1.5 on 783 (by digits); without top-p 117, 417 to 556; one row with
// top-p 85, 520.
#include "ops.hpp"

namespace sdlm {

namespace {

constexpr int TH = 1024;
typedef unsigned long long u64;
constexpr double ONE = 17592186044416.0;   // 2^44
constexpr double LOG2E = 1.4426950408889634;
constexpr uint32_t KEY_NEG_INF = 0x007fffffu, KEY_INF = 0xff800000u;

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
        return y >= -46.0 ? (u64)(exp2(y) * ONE + 0.5) : 0ull;   // nothing either where both are infinite, the largest logit and the temperature
    }
};

// What a search found: the token's key, how many of the tokens with that key come up to it (1: the first), count and weight of the order up to and including it.
struct Found { uint32_t key; int rank; u64 mass; };

struct Shared {
    u64 mass[2048];
    uint32_t cnt[2048];
    u64 red[TH / 64];
    double table[64];   // 2^(j / 64)
    Found f;
    u64 w;
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
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift - 10) {   // digits of 11, 11 and 10 bits: wide ones, so that the lanes of a wavefront seldom meet in one
        const int bits = shift == 0 ? 10 : 11, digits = 1 << bits, per = digits / 64;
        for (int i = tid; i < digits; i += TH) { sh.mass[i] = 0; sh.cnt[i] = 0; }
        __syncthreads();
        const uint32_t prefix = sh.prefix;
        for (int i = tid; i < row.V; i += TH) {
            const float z = row.at(i);
            const uint32_t k = key_of(z);
            if (z == -INFINITY || (shift < 21 && (k >> (shift + bits)) != prefix)) continue;
            atomicAdd(&sh.cnt[(k >> shift) & (digits - 1)], 1u);
            if (by != BY_COUNT) atomicAdd(&sh.mass[(k >> shift) & (digits - 1)], w(z));
        }
        __syncthreads();
        if (tid < 64) {   // lane l: `per` digits, from the highest down
            const int top = digits - 1 - per * tid;
            u64 m = 0, n = 0;
            for (int i = 0; i < per; ++i) { m += sh.mass[top - i]; n += sh.cnt[top - i]; }
            u64 ms = m, ns = n;
            for (int o = 1; o < 64; o <<= 1) {
                const u64 x = __shfl_up(ms, o), y = __shfl_up(ns, o);
                if (tid >= o) { ms += x; ns += y; }
            }
            ms += sh.acc_mass; ns += sh.acc_cnt;
            auto past = [&](u64 mass, u64 count) { return by == BY_COUNT ? count >= bound : by == MASS_AT_LEAST ? mass >= bound : mass > bound; };
            u64 lanes = __ballot(n && past(ms, ns));
            if (!lanes) lanes = 1ull << (63 - __clzll((long long)__ballot(n != 0)));   // not passed: the last token
            if (tid == __ffsll(lanes) - 1) {
                u64 mb = ms - m, nb = ns - n, ml = mb, nl = nb;
                int last = 0;
                for (int i = 0; i < per; ++i) {
                    if (!sh.cnt[top - i]) continue;
                    last = i; ml = mb; nl = nb;
                    mb += sh.mass[top - i]; nb += sh.cnt[top - i];
                    if (past(mb, nb)) break;
                }
                sh.prefix = prefix << bits | (uint32_t)(top - last);
                sh.acc_mass = ml; sh.acc_cnt = nl;
            }
        }
        __syncthreads();
    }
    u64 above = sh.acc_mass;
    if (by == BY_COUNT) {   // the weight in front of the key, which the counts did not need
        above = 0;
        for (int i = tid; i < row.V; i += TH) {
            const float z = row.at(i);
            if (key_of(z) > sh.prefix) above += w(z);
        }
        above = block_reduce(sh, above, [](u64 x, u64 y) { return x + y; });
    }
    if (tid == 0) {
        const uint32_t ties = sh.cnt[sh.prefix & 1023];
        const u64 each = w(of_key(sh.prefix)), m = above;
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

// The row by digits: right for every row, and slow.
template <typename T>
__device__ void by_digits(Shared &sh, const Row<T> &row, float M, float t, int k, float p, float mp, float u, int *id, float *prob)
{
    const Weigh w{(double)M, LOG2E / (double)t};
    auto add = [](u64 x, u64 y) { return x + y; };
    u64 n = 0, m = 0, mm = 0;
    const double least = (double)mp * ONE;
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
    const u64 at = (u64)(fmin(fmax((double)u, 0.0), 1.0) * (double)kept);
    const Found f = search(sh, row, w, MASS_ABOVE, min(at, kept - 1));
    *id = index_of(sh, row, f.key, f.rank);
    *prob = (float)((double)w(of_key(f.key)) / (double)kept);
}

// ------------------------------------------------------------------------------------------------ first launch
constexpr int PER_THREAD = 64, CHUNK = 256 * PER_THREAD;   // logits of a thread and of a workgroup
constexpr int RUNS = 9;                        // runs of a thread of the second launch, at most: the largest vocabulary has (524288 + 7) / 64
constexpr int OCTAVES = 24, PER_OCTAVE = 32, BINS = OCTAVES * PER_OCTAVE, COPIES = 4;   // the last bin, BINS: all below
constexpr int TOP_MAX = 2048;                  // largest top-k whose bound is taken from the runs of a long row: beyond, so many logits reach it that they cannot be held
constexpr double Y_MAX = 16384.0;              // largest exponent (of 2) whose fraction keeps 39 bits

// What a row's settings ask of the first launch.
__device__ inline bool wants_weights(const sdlm_sample_args &a, int r)
{
    const float t = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    return t > 0.f && !(mp > 1.f) && (k <= 0 || k >= a.vocab) && !(mp > 0.f && !(p < 1.f));
}

// ... of which min-p needs the sum alone.
__device__ inline bool wants_sum(const sdlm_sample_args &a, int r) { return a.min_p && a.min_p[r] > 0.f; }

// The row's 16-byte pieces: piece v holds elements [v E - lead, v E - lead + E), E to a piece; lead elements of the first lie in front of the row.
template <typename T>
struct Pieces {
    static constexpr int E = 16 / sizeof(T);
    const T *z;
    int V, lead;
    __device__ Pieces(const sdlm_sample_args &a, int r)
    {
        z = (const T *)a.logits + (size_t)r * a.row_stride;
        V = a.vocab;
        lead = (int)(((uintptr_t)z & 15) / sizeof(T));
    }
    // Piece v as it lies in memory; outside the row -infinity, and nothing outside it is read.
    __device__ uint4 raw(int v) const
    {
        const int i0 = v * E - lead;
        if (i0 >= 0 && i0 + E <= V) return *(const uint4 *)(z + i0);
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
            for (int e = k * E / 4; e < (k + 1) * E / 4; ++e)
                if (i0 + e >= 0 && i0 + e < V) {
                    if constexpr (sizeof(T) == 4) w[k] = __float_as_uint(z[i0 + e]);
                    else w[k] = e & 1 ? (w[k] & 0xffffu) | (uint32_t)z[i0 + e] << 16 : (w[k] & 0xffff0000u) | z[i0 + e];
                }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ void bare(const uint4 &u, float (&x)[E])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(w[e]);
            else x[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        }
    }
    static __device__ void values(const uint4 &u, float (&x)[E])
    {
        bare(u, x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = canon(x[e]);
    }
};

__host__ __device__ inline int n_chunks(int vocab, int esz) { return (vocab + 16 / esz - 1 + CHUNK - 1) / CHUNK; }

// Runs into which a thread's logits are divided, each with a maximum of its own: as many as the second launch can hold, so that also in small vocabularies there are
// more runs than candidates are asked for.
template <typename T>
__host__ __device__ inline int runs_of(int chunks)
{
    int n = PER_THREAD * (int)sizeof(T) / 16;
    while (n > 1 && chunks * n * 256 > TH * RUNS) n >>= 1;
    return n;
}

struct SampleWs {
    uint32_t *top;   // [row][chunk][run of a thread][256]: key of the largest logit of the run
    int32_t *ref;    // [row][chunk]: the power of two that the chunk's weights are relative to; NONE: no weights
    u64 *hist;       // [row][chunk][BINS + 1]
};
constexpr int NONE = -(1 << 30);

// The exponent of 2 of a logit's weight, rounded by itself: both launches have to find the same one, so it is no part of a fused product and sum.
__device__ inline double exponent(float z, double cs)
{
    double y = (double)z * cs;
    asm("" : "+v"(y));
    return y;
}

// 2^d in units of 2^-44, d <= 0: a table of 2^(j / 64) and a cubic for the rest, which depend on d's fraction alone.  The cubic's four fp32
// roundings are 2^-24 of |r| <= ln 2 / 128 each, its remainder r^4 / 24 and the result's last bit 2^-31: together below 2^-29 (largest found over 4e7 values: 2^-29.5).  So equal logits have equal weights whatever power of two they
// are held against, in both launches, and sums of weights down to 2^-14 of the largest are exact: a bound that falls between equal logits falls between the same ones as in the definition.
__device__ inline u64 fast_weight(double d, const double *table)
{
    const double magic = 6755399441055744.0;   // 1.5 2^52: the sum's low bits are the rounded integer
    const double s = d * 64.0 + magic;
    const int n = __double2loint(s);
    const float r = (float)(d - (s - magic) * (1.0 / 64.0)) * 0.69314718056f;   // |r| <= ln 2 / 128
    const float q = r * fmaf(r, fmaf(r, 0.16666667f, 0.5f), 1.f);
    const double t = table[n & 63];
    const uint32_t m = (uint32_t)__double2loint(fma(t, (double)q, t) + 6291456.0);   // + 1.5 2^22: an ulp of the sum is 2^-30
    return ((((u64)m << 15) >> -(n >> 6)) + 1) >> 1;
}

__device__ inline int bin_of(double y) { return (int)floor(y * -(double)PER_OCTAVE); }   // absolute: bin - PER_OCTAVE ref counts from the reference

template <typename T>
__global__ __launch_bounds__(256) void sample_scan_k(sdlm_sample_args a, SampleWs ws, int chunks)
{
    constexpr int E = Pieces<T>::E, N = PER_THREAD / E;
    const int r = blockIdx.x / chunks, c = blockIdx.x % chunks, tid = threadIdx.x;
    const Pieces<T> row(a, r);
    const bool weigh = wants_weights(a, r);
    float x[N][E], top_of[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        row.values(row.raw(c * (CHUNK / E) + i * 256 + tid), x[i]);
        top_of[i] = x[i][0];
#pragma unroll
        for (int e = 1; e < E; ++e) top_of[i] = fmaxf(top_of[i], x[i][e]);
    }
    const int per = runs_of<T>(chunks);
    uint32_t *keys = ws.top + ((size_t)r * chunks + c) * per * 256 + tid;
#pragma unroll
    for (int n = N; n >= 1; n >>= 1) {
        if (per == n)
#pragma unroll
            for (int i = 0; i < n; ++i) keys[i * 256] = key_of(top_of[i]);
#pragma unroll
        for (int i = 0; i < n / 2; ++i) top_of[i] = fmaxf(top_of[2 * i], top_of[2 * i + 1]);
    }
    if (!weigh) return;
    float mx = top_of[0];
    __shared__ double table[64];
    __shared__ u64 hist[COPIES][BINS + 1];
    __shared__ float red[4];
    const bool sum = wants_sum(a, r);
    if (tid < 64) table[tid] = exp2(tid * (1.0 / 64.0));
    for (int i = tid; i < COPIES * (BINS + 1); i += 256) (&hist[0][0])[i] = 0;
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const double cs = LOG2E / (double)(a.temperature ? a.temperature[r] : 1.f), top = (double)mx * cs;
    const bool usable = top > -Y_MAX && top < Y_MAX;
    const int ref = usable ? (int)ceil(top) : NONE;
    if (tid == 0) ws.ref[(size_t)r * chunks + c] = ref;
    if (!usable) return;
    u64 rest = 0, *mine = hist[tid % COPIES];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const double y = exponent(x[i][e], cs), d = y - ref;
            if (!(d > -46.0)) continue;
            const u64 w = fast_weight(d, table);
            const int b = sum ? BINS : bin_of(y) + PER_OCTAVE * ref;
            if (b < BINS) atomicAdd(&mine[max(b, 0)], w);
            else rest += w;
        }
    if (rest) atomicAdd(&mine[BINS], rest);
    __syncthreads();
    u64 *out = ws.hist + ((size_t)r * chunks + c) * (BINS + 1);
    for (int i = sum ? BINS + tid : tid; i <= BINS; i += 256) {
        u64 v = 0;
#pragma unroll
        for (int k = 0; k < COPIES; ++k) v += hist[k][i];
        out[i] = v;
    }
}

// ------------------------------------------------------------------------------------------------ second launch
constexpr int CAND = 4096;             // candidates that are sorted

struct Lists {
    u64 cand[CAND];                    // key << 32 | ~index: descending order is the row's order
    u64 cum[CAND];                     // weights, running or single
    u64 part[TH];                      // the candidates of one fine bin
    u64 mass[TH];                      // fine bins: weights and counts
    uint32_t cnt[TH];
    uint16_t run[TH * RUNS];           // runs that may hold candidates
    int n_cand, n_run, n_part;
};

// Exclusive prefix sum over the workgroup, and the sum.
__device__ inline u64 block_scan(Shared &sh, u64 v, u64 *sum)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 x = v;
    for (int o = 1; o < 64; o <<= 1) { const u64 y = __shfl_up(x, o); if (lane >= o) x += y; }
    __syncthreads();
    if (lane == 63) sh.red[wave] = x;
    __syncthreads();
    u64 before = 0, s = 0;
    for (int i = 0; i < TH / 64; ++i) { if (i < wave) before += sh.red[i]; s += sh.red[i]; }
    *sum = s;
    return before + x - v;
}

// A lower bound of the k-th largest run maximum, by its upper 22 bits (0 if there are fewer runs): the few candidates that it lets in besides cost less than the third pass.
__device__ uint32_t kth_run(Shared &sh, const uint32_t (&keys)[RUNS], int k)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    int want = k;
    for (int shift = 21; shift >= 10; shift -= 11) {
        for (int i = tid; i < 2048; i += TH) sh.cnt[i] = 0;
        if (tid == 0) sh.hit = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < RUNS; ++j)
            if (keys[j] && (shift == 21 || (keys[j] >> 21) == prefix)) atomicAdd(&sh.cnt[(keys[j] >> shift) & 2047], 1u);
        __syncthreads();
        const int d = 2047 - 2 * tid, c0 = (int)sh.cnt[d], c1 = (int)sh.cnt[d - 1];   // two digits a thread, from the highest down
        u64 all;
        const int before = (int)block_scan(sh, c0 + c1, &all);
        if (before < want && before + c0 + c1 >= want) {
            const bool first = before + c0 >= want;
            sh.prefix = (shift == 21 ? 0u : prefix << 11) | (uint32_t)(first ? d : d - 1);
            sh.hit = want - before - (first ? 0 : c0);
        }
        __syncthreads();
        want = sh.hit;
        if (want == 0) return 0;
        prefix = sh.prefix;
        __syncthreads();
    }
    return prefix << 10;
}

// The smallest key in [k0, k1] whose logit lies in bin `bin` (absolute) or in a heavier one; k1 + 1 if there is none.  By a wavefront: bins do not rise with the logit.
__device__ uint32_t first_of_bin(uint32_t k0, uint32_t k1, int bin, double cs)
{
    uint32_t n = k1 - k0 + 1;
    while (n > 1) {
        const uint32_t step = (n + 63) / 64, at = step * ((threadIdx.x & 63) + 1) - 1;
        const int first = __ffsll(__ballot(at >= n - 1 || bin_of(exponent(of_key(k0 + at), cs)) <= bin)) - 1;
        k0 += step * first;
        n = min(step, n - step * first);
    }
    return bin_of(exponent(of_key(k0), cs)) <= bin ? k0 : k0 + 1;
}

// Candidates: the logits whose key is at least `lo` and at most `hi`, from the runs whose maximum is at least lo.  Returns whether they fit.
template <typename T>
__device__ bool gather(Lists &ls, const Pieces<T> &row, const uint32_t (&keys)[RUNS], int per, uint32_t lo, uint32_t hi)
{
    constexpr int E = Pieces<T>::E, N = PER_THREAD / E;
    const int lp = 31 - __clz(per), lg = 31 - __clz(N) - lp;   // log2 of the runs of a thread of the first launch, and of a run's pieces
    if (threadIdx.x == 0) { ls.n_cand = 0; ls.n_run = 0; }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < RUNS; ++j)
        if (keys[j] >= lo && keys[j] > KEY_NEG_INF) ls.run[atomicAdd(&ls.n_run, 1)] = (uint16_t)(threadIdx.x + j * TH);
    __syncthreads();
    // Bound by its instructions: a unit has a workgroup for all of a row's logits where the bound is low.  So two pieces of a run are one trip, a logit costs two comparisons and a bit, and the rest
    // is done for those that pass (few), a thread's one behind the other.  A wavefront takes room for all of its trip's candidates with one atomic.
    const bool two = lg > 0;
    const int l2 = two ? lg - 1 : 0, trips = ls.n_run << l2;
    const float least = of_key(max(lo, KEY_NEG_INF + 1)), most = of_key(min(hi, KEY_INF));
    for (int q = threadIdx.x; q < trips; q += TH) {
        const int run = ls.run[q >> l2], v = (((run >> 8) << lg) + ((q & ((1 << l2) - 1)) << (lg - l2))) * 256 + (run & 255), i0 = v * E - row.lead;
        const uint4 raw0 = row.raw(v), raw1 = two ? row.raw(v + 256) : make_uint4(0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu);   // not numbers: in no bound
        float x[E], y[E];
        row.bare(raw0, x);
        row.bare(raw1, y);
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            hits |= x[e] >= least && x[e] <= most ? 1u << e : 0u;
            hits |= y[e] >= least && y[e] <= most ? 1u << (E + e) : 0u;
        }
        if (!__any(hits)) continue;
        const int n = __popc(hits);
        int before = 0, total = 0;
#pragma unroll
        for (int k = 1; k <= 2 * E; k <<= 1) {
            const u64 w = __ballot(n & k);
            before += k * (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(w >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)w, 0));
            total += k * __popcll(w);
        }
        int at = 0;
        const int leader = __ffsll(__ballot(1)) - 1;
        if ((threadIdx.x & 63) == leader) at = atomicAdd(&ls.n_cand, total);
        at = __builtin_amdgcn_readfirstlane(at) + before;
        for (; hits; hits &= hits - 1, ++at) {
            const int e = __ffs((int)hits) - 1, i = i0 + e + (e >= E ? 255 * E : 0);
            if (at < CAND) ls.cand[at] = (u64)key_of(canon(to_f<T>(row.z[i]))) << 32 | (uint32_t)~(uint32_t)i;
        }
    }
    __syncthreads();
    return ls.n_cand <= CAND;
}

// Sort n entries in descending order; with room up to the next power of two.
__device__ void sort(u64 *v, int n)
{
    const int tid = threadIdx.x;
    if (n <= 128) {   // every entry counts those in front of it
        u64 x = 0;
        int rank = 0;
        if (tid < n) {
            x = v[tid];
            for (int i = 0; i < n; ++i) rank += v[i] > x;
        }
        __syncthreads();
        if (tid < n) v[rank] = x;
        __syncthreads();
        return;
    }
    int p = 256;
    while (p < n) p <<= 1;
    for (int i = n + tid; i < p; i += TH) v[i] = 0;
    __syncthreads();
    for (int k = 2; k <= p; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int i = tid; i < p / 2; i += TH) {
                const int x = 2 * i - (i & (j - 1)), y = x + j;
                const u64 f = v[x], g = v[y];
                if ((f < g) == ((x & k) == 0)) { v[x] = g; v[y] = f; }
            }
            __syncthreads();
        }
}

// The first of n candidates whose running weight is at least (above) `bound`; n if there is none.
__device__ int first_past(const Lists &ls, int n, u64 bound, bool above)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (above ? ls.cum[mid] > bound : ls.cum[mid] >= bound) hi = mid; else lo = mid + 1;
    }
    return lo;
}

__device__ inline int index_at(const Lists &ls, int i) { return (int)~(uint32_t)ls.cand[i]; }
__device__ inline float logit_at(const Lists &ls, int i) { return of_key((uint32_t)(ls.cand[i] >> 32)); }

struct Weight {   // against a power of two, as the first launch has it, or against the largest (table: null); one type, so that what takes weights is there once
    double cs, ref;
    const double *table;
    __device__ u64 operator()(float z) const
    {
        if (!table) return Weigh{ref, cs}(z);
        const double d = exponent(z, cs) - ref;
        return d > -46.0 ? fast_weight(d, table) : 0ull;
    }
};

// Running weights of the first n candidates, starting at `base`.
__device__ void weigh(Shared &sh, Lists &ls, int n, u64 base, const Weight &w)
{
    for (int i0 = 0; i0 < n; i0 += TH) {
        const int i = i0 + threadIdx.x;
        const u64 x = i < n ? w(of_key((uint32_t)(ls.cand[i] >> 32))) : 0;
        u64 all;
        const u64 before = base + block_scan(sh, x, &all);
        if (i < n) ls.cum[i] = before + x;
        base += all;
    }
    __syncthreads();
}

// Many candidates are not sorted: they go into TH bins by their key, a thread a bin, and only the bin in which a bound is passed is (4000 candidates: 8 us a bound instead of 30 for
// all).  base: weight in front of the first candidate.
struct Picked { u64 mass, w; int index; };   // weight up to and with the candidate, its own, its place in the row

struct Fine {
    Shared &sh;
    Lists &ls;
    const Weight &w;
    int n, shift;
    uint32_t hi;
    u64 m, m_before;
    int c, c_before;
    __device__ int bin(u64 cand) const { return (int)((hi - (uint32_t)(cand >> 32)) >> shift); }
    __device__ Fine(Shared &sh_, Lists &ls_, const Weight &w_, int n_, u64 base) : sh(sh_), ls(ls_), w(w_), n(n_)
    {
        const int tid = threadIdx.x;
        uint32_t h = 0, l = 0xffffffffu;
        for (int i = tid; i < n; i += TH) { const uint32_t k = (uint32_t)(ls.cand[i] >> 32); h = max(h, k); l = min(l, k); }
        hi = (uint32_t)block_reduce(sh, h, [](u64 x, u64 y) { return x > y ? x : y; });
        const uint32_t lo = (uint32_t)block_reduce(sh, l, [](u64 x, u64 y) { return x < y ? x : y; });
        const int bits = 32 - __clz((int)(hi - lo));
        shift = bits > 10 ? bits - 10 : 0;
        ls.mass[tid] = 0; ls.cnt[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += TH) {
            const u64 v = ls.cand[i];
            atomicAdd(&ls.mass[bin(v)], w(of_key((uint32_t)(v >> 32))));
            atomicAdd(&ls.cnt[bin(v)], 1u);
        }
        __syncthreads();
        u64 all;
        m = ls.mass[tid]; c = (int)ls.cnt[tid];
        m_before = base + block_scan(sh, m, &all);
        c_before = (int)block_scan(sh, c, &all);
    }
    // The first candidate by which the running count or weight passes `bound` (the last one if none does); false: its bin is too full.
    __device__ bool pick(int by, u64 bound, Picked *p)
    {
        const int tid = threadIdx.x;
        __syncthreads();
        if (tid == 0) { sh.hit = -1; ls.n_part = 0; }
        __syncthreads();
        const u64 x0 = by == BY_COUNT ? c_before : m_before, x1 = by == BY_COUNT ? c_before + c : m_before + m;
        auto past = [&](u64 x) { return by == MASS_ABOVE ? x > bound : x >= bound; };
        if (c && past(x1) && !past(x0)) { sh.hit = tid; sh.acc_mass = m_before; sh.acc_cnt = c_before; }
        __syncthreads();
        if (sh.hit < 0) {   // none: the last candidate's bin
            const int last = (int)block_reduce(sh, c ? tid : 0, [](u64 x, u64 y) { return x > y ? x : y; });
            if (tid == last) { sh.hit = tid; sh.acc_mass = m_before; sh.acc_cnt = c_before; }
            __syncthreads();
        }
        const int b = sh.hit;
        for (int i = tid; i < n; i += TH) {
            const u64 v = ls.cand[i];
            if (bin(v) != b) continue;
            const int at = atomicAdd(&ls.n_part, 1);
            if (at < TH) ls.part[at] = v;
        }
        __syncthreads();
        const int np = ls.n_part;
        if (np > TH) return false;
        sort(ls.part, np);
        const u64 v = tid < np ? ls.part[tid] : 0, x = tid < np ? w(of_key((uint32_t)(v >> 32))) : 0;
        u64 all;
        const u64 before = sh.acc_mass + block_scan(sh, x, &all), seen = sh.acc_cnt + tid;
        const bool first = by == BY_COUNT ? seen + 1 == bound : past(before + x) && !past(before);
        const u64 any = __syncthreads_or(tid < np && first);
        if (tid < np && (any ? first : tid == np - 1)) { sh.f.mass = before + x; sh.w = x; sh.f.rank = (int)~(uint32_t)v; }
        __syncthreads();
        *p = Picked{sh.f.mass, sh.w, sh.f.rank};
        return true;
    }
};
constexpr int SORT_ALL = 128;          // candidates that are simply sorted

template <typename T>
__global__ __launch_bounds__(TH) void sample_draw_k(sdlm_sample_args a, SampleWs ws, int chunks)
{
    __shared__ Shared sh;
    __shared__ Lists ls;
    const int r = blockIdx.x, tid = threadIdx.x, per = runs_of<T>(chunks), runs = chunks * per * 256;
    const Pieces<T> row(a, r);
    const Row<T> plain{row.z, row.V};
    uint32_t keys[RUNS], kmax = 0;
#pragma unroll
    for (int j = 0; j < RUNS; ++j) {
        keys[j] = tid + j * TH < runs ? ws.top[(size_t)r * runs + tid + j * TH] : 0;
        kmax = max(kmax, keys[j]);
    }
    const float t = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f, u = a.u[r];
    const int k = a.top_k ? a.top_k[r] : 0;
    kmax = (uint32_t)block_reduce(sh, kmax, [](u64 x, u64 y) { return x > y ? x : y; });
    const float M = of_key(kmax);
    int id = -1;
    float prob = 0.f;
    bool done = true;
    const double cs = LOG2E / (double)t, share = fmin(fmax((double)u, 0.0), 1.0);
    const bool top_k = k > 0 && k < row.V;
    if (M == -INFINITY) {
        // every token is masked
    } else if (!(t > 0.f) || mp > 1.f) {   // the first token: no weight reaches a min_p above 1
        if ((done = gather(ls, row, keys, per, kmax, kmax))) {
            u64 best = 0;
            for (int i = tid; i < ls.n_cand; i += TH) best = max(best, ls.cand[i]);
            id = (int)~(uint32_t)block_reduce(sh, best, [](u64 x, u64 y) { return x > y ? x : y; });
        } else { id = index_of(sh, plain, kmax, 1); done = true; }
        prob = 1.f;
    } else if (top_k || mp > 0.f) {
        // candidates are a first part of the order that holds everything that can be kept
        const Weigh exact{(double)M, cs};
        const bool by_min = !top_k;
        uint32_t lo;
        u64 row_mass = 0;   // by_min and top_p, which is a share of the whole row: its weight, and what that is held against
        int ref = 0;
        if (by_min) {
            const double z = (double)M + (double)t * log((double)mp);
            lo = M == INFINITY ? kmax : t == INFINITY ? 0 : key_of((float)(z - (fabs(z) + fabs((double)M)) * 1e-6 - 1e-30));   // a little below: the weights decide
            if (p < 1.f) {
                const double top = (double)M * cs;
                done = fabs(top) < Y_MAX - 64.0;
                if (done) {
                    if (tid < 64) sh.table[tid] = exp2(tid * (1.0 / 64.0));
                    ref = (int)ceil(top);
                    for (int c = tid; c < chunks; c += TH) {
                        const int back = ref - ws.ref[(size_t)r * chunks + c];
                        if (back < 46) row_mass += ws.hist[((size_t)r * chunks + c) * (BINS + 1) + BINS] >> back;
                    }
                    row_mass = block_reduce(sh, row_mass, [](u64 x, u64 y) { return x + y; });
                }
            }
        } else {
            done = k <= CAND;
            lo = k <= TOP_MAX || row.V <= CAND ? kth_run(sh, keys, k) : KEY_INF + 1;
        }
        if (done) {
            done = lo <= KEY_INF && gather(ls, row, keys, per, lo, KEY_INF);
            if (!done && top_k) {   // too few runs for a bound (a short row, or few tokens above -infinity), or too many equal logits near it: the k-th itself
                __syncthreads();
                done = gather(ls, row, keys, per, search(sh, plain, exact, BY_COUNT, (u64)k).key, KEY_INF);
            }
        }
        if (done) {
            const bool shares = by_min && p < 1.f;
            const Weight w{cs, shares ? (double)ref : (double)M, shares ? sh.table : nullptr};   // of the sums; a single weight against min_p is always the exact one
            int n = ls.n_cand;
            const double least = (double)mp * ONE;
            double total = (double)row_mass;
            bool fine = n > SORT_ALL;
            if (fine) {
                Fine bins(sh, ls, w, n, 0);
                Picked at;
                u64 kept = ~0ull, heavy = 0;
                if (top_k && k < n) { fine = bins.pick(BY_COUNT, (u64)k, &at); kept = at.mass; }
                else { u64 all; block_scan(sh, bins.m, &all); kept = all; }
                if (top_k) total = (double)kept;
                if (fine && p < 1.f) {
                    const u64 bound = (u64)fmin(ceil(fmax((double)p, 0.0) * total), 1.8e19);
                    if (bound <= kept) { fine = bins.pick(MASS_AT_LEAST, max(bound, (u64)1), &at); kept = at.mass; }
                }
                if (fine && mp > 0.f) {
                    for (int i = tid; i < n; i += TH) { const float z = logit_at(ls, i); const u64 x = w(z); heavy += (double)(shares ? exact(z) : x) >= least ? x : 0; }
                    kept = min(kept, block_reduce(sh, heavy, [](u64 x, u64 y) { return x + y; }));
                }
                if (fine && (fine = bins.pick(MASS_ABOVE, min((u64)(share * (double)kept), kept - 1), &at))) {
                    id = at.index;
                    prob = (float)((double)at.w / (double)kept);
                }
            }
            if (!fine) {
                __syncthreads();
                sort(ls.cand, n);
                if (top_k) n = min(n, k);
                weigh(sh, ls, n, 0, w);
                if (top_k) total = (double)ls.cum[n - 1];
                int keep = n;
                if (p < 1.f) keep = min(n, 1 + first_past(ls, n, (u64)fmin(ceil(fmax((double)p, 0.0) * total), 1.8e19), false));
                if (mp > 0.f) {   // weights fall along the order: the first that is too light ends it
                    int l = 1, h = keep;
                    while (l < h) {
                        const int mid = (l + h) >> 1;
                        if ((double)(shares ? exact(logit_at(ls, mid)) : ls.cum[mid] - ls.cum[mid - 1]) < least) h = mid; else l = mid + 1;
                    }
                    keep = h;
                }
                const u64 kept = ls.cum[keep - 1];
                const int at = first_past(ls, keep, min((u64)(share * (double)kept), kept - 1), true);
                id = index_at(ls, at);
                prob = (float)((double)(ls.cum[at] - (at ? ls.cum[at - 1] : 0)) / (double)kept);
            }
        }
    } else {
        // the whole row, by the histogram
        const double top = (double)M * cs;
        done = fabs(top) < Y_MAX - 64.0;
        if (done) {
            const int ref = (int)ceil(top);
            if (tid < 64) sh.table[tid] = exp2(tid * (1.0 / 64.0));
            const Weight w{cs, (double)ref, sh.table};
            u64 m = 0, rest = 0, all, rest_all;
            for (int c = tid; c < chunks; c += TH) sh.cnt[c] = (uint32_t)min(ref - ws.ref[(size_t)r * chunks + c], 46);   // octaves that a chunk's weights are moved down; 46: all of it
            __syncthreads();
            const u64 *hist = ws.hist + (size_t)r * chunks * (BINS + 1);
            if (tid < BINS)
#pragma unroll 5
                for (int c = 0; c < chunks; ++c) {
                    const int back = (int)sh.cnt[c], b = tid - PER_OCTAVE * back;
                    const u64 *h = hist + (size_t)c * (BINS + 1);
                    m += (b >= 0 && back < 46 ? h[b] : 0) >> back;
                    rest += (tid + PER_OCTAVE * back >= BINS && back < 46 ? h[tid] : 0) >> back;   // moved below the last bin
                }
            if (tid < chunks && sh.cnt[tid] < 46) rest += hist[(size_t)tid * (BINS + 1) + BINS] >> sh.cnt[tid];
            const u64 before = block_scan(sh, m, &all);
            block_scan(sh, rest, &rest_all);
            const u64 total = all + rest_all;
            // The bin in which the running weight passes `bound`, and the token of it that does.  A bin of tokens below 2^-14 of the largest may be summed otherwise than the tokens
            // one by one, so that a bound just below the weight that top_p keeps may seem to lie behind the cut's bin: it is the cut's token then, which *p holds.
            int cut = BINS;
            auto locate = [&](u64 bound, bool above, Picked *p) -> bool {
                if (tid == 0) sh.hit = -1;
                __syncthreads();
                const u64 end = before + m;
                if (tid < BINS && m && (above ? end > bound && before <= bound : end >= bound && before < bound)) { sh.hit = tid; sh.acc_mass = before; }
                __syncthreads();
                const int b = sh.hit;
                const u64 base = sh.acc_mass;
                __syncthreads();
                if (cut < BINS && (b < 0 || b > cut)) return true;
                if (b < 0) return false;   // among the lightest
                if (!above) cut = b;
                const int bin = b - PER_OCTAVE * ref;
                // logits of the bin, -bin / PER_OCTAVE >= y > -(bin + 1) / PER_OCTAVE, first a little widened, then as the first launch told them apart
                const double zh = -(double)bin / PER_OCTAVE / cs, zl = -(double)(bin + 1) / PER_OCTAVE / cs, wide = (fabs(zh) + fabs(zl)) * 1e-6 + 1e-30;
                const uint32_t k0 = max(key_of((float)(zl - wide)), KEY_NEG_INF + 1), k1 = min(key_of((float)(zh + wide)), KEY_INF - 1);
                if (k0 > k1) return false;
                if (tid < 128) {
                    const uint32_t k = first_of_bin(k0, k1, tid < 64 ? bin : bin - 1, cs);
                    if ((tid & 63) == 0) sh.cnt[tid >> 6] = k;
                }
                __syncthreads();
                const uint32_t lo = sh.cnt[0], hi = sh.cnt[1] - 1;
                if (!gather(ls, row, keys, per, lo, hi) || ls.n_cand == 0) return false;
                const int n = ls.n_cand;
                if (n > SORT_ALL) {
                    Fine bins(sh, ls, w, n, base);
                    if (bins.pick(above ? MASS_ABOVE : MASS_AT_LEAST, bound, p)) return true;
                    __syncthreads();
                }
                sort(ls.cand, n);
                weigh(sh, ls, n, base, w);
                const int at = min(first_past(ls, n, bound, above), n - 1);   // (as above) at most the last
                *p = Picked{ls.cum[at], w(logit_at(ls, at)), index_at(ls, at)};
                return true;
            };
            u64 kept = total;
            Picked at;
            if (p < 1.f) {
                done = locate(max((u64)ceil(fmax((double)p, 0.0) * (double)total), (u64)1), false, &at);
                kept = at.mass;
                __syncthreads();
            }
            if (done && (done = locate(min((u64)(share * (double)kept), kept - 1), true, &at))) {
                id = at.index;
                prob = (float)((double)at.w / (double)kept);
            }
        }
    }
    if (!done) {
        __syncthreads();
        by_digits(sh, plain, M, t, k, p, mp, u, &id, &prob);
    }
    if (tid == 0) {
        a.ids[r] = id;
        if (a.prob) a.prob[r] = prob;
    }
}

SampleWs sample_ws(int rows, int vocab, void *workspace, size_t *bytes)
{
    const size_t n = (size_t)rows * n_chunks(vocab, 2);   // bf16 rows may begin further in front
    char *w = (char *)workspace;
    SampleWs s;
    size_t o = 0;
    auto take = [&](size_t b) { char *at = w + o; o += (b + 255) / 256 * 256; return at; };
    s.top = (uint32_t *)take((size_t)rows * TH * RUNS * 4);
    s.ref = (int32_t *)take(n * 4);
    s.hist = (u64 *)take(n * (BINS + 1) * 8);
    *bytes = o;
    return s;
}

template <typename T>
void sample_t(hipStream_t s, const sdlm_sample_args &a, const SampleWs &ws)
{
    const int chunks = n_chunks(a.vocab, sizeof(T));
    hipLaunchKernelGGL(sample_scan_k<T>, dim3((unsigned)a.rows * chunks), dim3(256), 0, s, a, ws, chunks);
    hipLaunchKernelGGL(sample_draw_k<T>, dim3(a.rows), dim3(TH), 0, s, a, ws, chunks);
}

}  // namespace

bool sample_fits(int rows, int vocab) { return rows <= SAMPLE_MAX_ROWS && (double)rows * n_chunks(vocab, 2) < (double)(1 << 24); }   // threads of a launch fit 32 bits

size_t sample_workspace_bytes(int rows, int vocab)
{
    size_t n;
    sample_ws(rows > 0 ? rows : 1, vocab, nullptr, &n);
    return n;
}

void launch_sample(hipStream_t s, const sdlm_sample_args &a, void *workspace)
{
    size_t n;
    const SampleWs ws = sample_ws(a.rows, a.vocab, workspace, &n);
    if (a.dtype == 0) sample_t<float>(s, a, ws); else sample_t<bf16_t>(s, a, ws);
}

}  // namespace sdlm
