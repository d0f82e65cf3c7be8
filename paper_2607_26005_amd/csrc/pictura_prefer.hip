// A preference loss over pairs of sequences of decisions, and its gradient.
//
// Per row l = log softmax(x)[action]; per sequence D = sum (l - ref) over its rows (or their
// mean); per pair m = beta (D_preferred - D_other) and
//     loss = -(1 - eps) log sigmoid(m) - eps log sigmoid(-m),
//     dloss/dx_i = +-c (delta_ia - p_i),  c = w beta (eps sigmoid(m) - (1 - eps) sigmoid(-m)),
// for the rows of the preferred sequence (+) and the other (-).  A row's gradient hangs on
// all rows of its pair.
//
// Heads of up to 64 actions: a workgroup to a pair, which keeps its rows in registers
// between the sums and the gradient (pairs of more than 256 rows of 16 actions, or 32 of 64,
// read them again; pairs of thousands of rows take the three launches of larger heads).
// Larger heads: one launch for the rows' log-probabilities, one for the pairs, one for the
// gradient, which reads the logits again, as a pair's rows do not fit on the chip.
//
// Measured (one MI355X): 1,024 pairs of 2 x 128 rows of 12, masked, 13.5 us and the statistics 3
// (31 MB, 6 us at a copy's rate: bound by the latencies from offsets to gradient); 2,879
// rows of 16,381 in bf16 23 us, 5 and 32 (94 MB read, then read and written: 4.2 and 5.9 TB/s,
// some of it from the caches).
#include <cmath>

#include "pictura.h"
#include "pictura_lanes.h"
#include "pictura_policy.h"

#pragma clang fp contract(off)

namespace pictura {
namespace {

template <int N>
struct Int {
    static constexpr int value = N;
};

struct Pairs {
    const int64_t* actions;
    const int64_t* offsets;   // [2 count + 1], of rows
    const float* ref;         // or null: zeros
    const float* weights;     // or null: ones
    int64_t count;
    float beta, smoothing, denominator;
    int32_t average;
    float* stats;
    float* ratios;            // [2 count]
    void* dlogits;
    int64_t dstride;
};

constexpr int kPairThreads = 256;       // of a workgroup that sums up a pair
constexpr int kTerms = 4;               // of a pair: loss, rewards, whether the preferred one's is larger
constexpr int64_t kFewPairs = 2048;     // weights of so many are added up by every workgroup that needs their sum

struct Scratch {
    double* omega;     // the sum of the weights, where there are more pairs than that
    double* terms;     // [count][kTerms], times the weight
    float2* softmax;   // [rows]: largest logit, 1 / sum of exponentials
    float* ratio;      // [rows]: l - ref
    float* factor;     // [rows]: 1 or 0 (whether the row counts), then its c
};

template <int G, class V>
__device__ __forceinline__ V group_sum(V x)
{
    if constexpr (G > 1) x = x + lanes<0xB1, 0xf>((V)0, x);
    if constexpr (G > 2) x = x + lanes<0x4E, 0xf>((V)0, x);
    if constexpr (G > 4) x = x + lanes<0x141, 0xf>((V)0, x);
    if constexpr (G > 8) x = x + lanes<0x140, 0xf>((V)0, x);
    if constexpr (G > 16) x = x + __shfl_xor(x, 16);
    if constexpr (G > 32) x = x + __shfl_xor(x, 32);
    return x;
}

template <int G>
__device__ __forceinline__ float group_max(float x)
{
    if constexpr (G > 1) x = fmaxf(x, lanes<0xB1, 0xf>(x, x));
    if constexpr (G > 2) x = fmaxf(x, lanes<0x4E, 0xf>(x, x));
    if constexpr (G > 4) x = fmaxf(x, lanes<0x141, 0xf>(x, x));
    if constexpr (G > 8) x = fmaxf(x, lanes<0x140, 0xf>(x, x));
    if constexpr (G > 16) x = fmaxf(x, __shfl_xor(x, 16));
    if constexpr (G > 32) x = fmaxf(x, __shfl_xor(x, 32));
    return x;
}

// exp(x - top), 0 for -inf; a NaN stays one.  top is finite, or infinite with a NaN to come.
// For 16-bit logits the product with log2 e is rounded once, off by up to 2^-24 of x - top:
// far below what their gradient's rounding takes.
template <class T>
__device__ __forceinline__ float weight_of(float x, float top)
{
    const float d = x - top;
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(d * kLog2e);
    return exp_of(d < -200.0f ? -200.0f : d);
}

// The rows of sequence s, [first, second), whatever the offsets say.
__device__ __forceinline__ int64_t bound_of(const Pairs& q, int64_t i, int64_t rows)
{
    const int64_t o = q.offsets[i];
    return o < 0 ? 0 : o > rows ? rows : o;
}

// This thread's part of the sum of the weights, where every workgroup adds them up.
template <int NT>
__device__ __forceinline__ double weight_part(const Pairs& q)
{
    double x = 0.0;
    if (q.weights && q.denominator == 0.0f && q.count <= kFewPairs)
        for (int64_t i = threadIdx.x; i < q.count; i += NT) x += (double)q.weights[i];
    return x;
}

// 1 / sum of the weights: of the pairs (sum: where every workgroup adds them up), given, or
// 0 where that is 0.
__device__ __forceinline__ double inverse_weight(const Pairs& q, const Scratch& k, double sum)
{
    if (q.denominator != 0.0f) sum = q.denominator;
    else if (!q.weights) sum = (double)q.count;
    else if (q.count > kFewPairs) sum = *k.omega;
    return sum != 0.0 ? 1.0 / sum : 0.0;
}

// What a pair's sums (of ratios and of rows that count) make of it.
struct PairTerms {
    double t[kTerms];
    double ratio[2];   // D of both
    float c[2];        // factor of their rows
};

__device__ __forceinline__ PairTerms pair_terms(const Pairs& q, int64_t p, const double (&sum)[2], const double (&rows)[2], double inverse)
{
    PairTerms r{};
    double part[2];
    for (int i = 0; i < 2; ++i) {
        part[i] = q.average && rows[i] > 1.0 ? 1.0 / rows[i] : 1.0;
        r.ratio[i] = sum[i] * part[i];
    }
    const double w = q.weights ? (double)q.weights[p] : 1.0;
    if (w == 0.0) return r;   // (its numbers are not looked at)
    const double beta = (double)q.beta, eps = (double)q.smoothing, m = beta * (r.ratio[0] - r.ratio[1]);
    // (fp32: these two are off by a few units, and all four waves' fp64 ones take 6 us)
    const float ef = expf(-(float)fabs(m));
    const double e = ef, near = log1pf(ef);                           // log sigmoid(-+m) = -(max(+-m, 0) + near)
    const double lose = fmax(-m, 0.0) + near, win = fmax(m, 0.0) + near;
    const double up = (m > 0.0 ? e : 1.0) / (1.0 + e), down = (m > 0.0 ? 1.0 : e) / (1.0 + e);   // sigmoid(-m), sigmoid(m)
    double loss = (1.0 - eps) * lose;
    if (eps > 0.0) loss += eps * win;
    if (m != m) loss = m;
    r.t[0] = w * loss;
    r.t[1] = w * (beta * r.ratio[0]);
    r.t[2] = w * (beta * r.ratio[1]);
    r.t[3] = m > 0.0 ? w : 0.0;
    const double c = m != m ? m : w * inverse * beta * (eps * down - (1.0 - eps) * up);
    r.c[0] = (float)(c * part[0]);
    r.c[1] = (float)(-c * part[1]);
    return r;
}

// Sum of the weights of many pairs, in a fixed order.
static __global__ __launch_bounds__(1024) void weight_sum_kernel(const Pairs q, const Scratch k)
{
    __shared__ double lds[16];
    double x = 0.0;
    for (int64_t i = threadIdx.x; i < q.count; i += 1024) x += (double)q.weights[i];
    x = block_sum<16>(x, lds);
    if (threadIdx.x == 0) *k.omega = x;
}

// Means of the pairs' terms, by one workgroup of NT threads.
template <int NT>
__device__ void write_stats(const Pairs& q, const Scratch& k)
{
    __shared__ double lds[NT / 64][kTerms + 1];
    double t[kTerms + 1] = {};
    for (int64_t i = threadIdx.x; i < q.count; i += NT) {
#pragma unroll
        for (int j = 0; j < kTerms; ++j) t[j] += k.terms[i * kTerms + j];
    }
    t[kTerms] = weight_part<NT>(q);
#pragma unroll
    for (int j = 0; j <= kTerms; ++j) {
        t[j] = wave_sum(t[j]);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6][j] = t[j];
    }
    __syncthreads();
    if (threadIdx.x < kTerms) {
        double x = 0.0, w = 0.0;
        for (int i = 0; i < NT / 64; ++i) {
            x += lds[i][threadIdx.x];
            w += lds[i][kTerms];
        }
        q.stats[threadIdx.x] = (float)(x * inverse_weight(q, k, w));
    }
}

static __global__ __launch_bounds__(256) void stats_kernel(const Pairs q, const Scratch k) { write_stats<256>(q, k); }

// The sums of a pair over a workgroup of four waves, its terms by the first wave, and the
// factors of its rows for all: two barriers.
__device__ __forceinline__ void finish_pair(const Pairs& q, const Scratch& k, int64_t p, const double (&sum)[2],
                                            const uint32_t (&rows)[2], float (&c)[2])
{
    __shared__ double parts[4][5];
    __shared__ float factors[2];
    const int wave = threadIdx.x >> 6;
    const double t[5] = {wave_sum(sum[0]), wave_sum(sum[1]), (double)wave_sum(rows[0]), (double)wave_sum(rows[1]),
                         wave_sum(weight_part<256>(q))};
    __syncthreads();   // (what stands there may still be read from before)
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int j = 0; j < 5; ++j) parts[wave][j] = t[j];
    }
    __syncthreads();
    if (wave == 0) {
        double x[5];
#pragma unroll
        for (int j = 0; j < 5; ++j) x[j] = ((parts[0][j] + parts[1][j]) + parts[2][j]) + parts[3][j];
        const double all[2] = {x[0], x[1]}, count[2] = {x[2], x[3]};
        const PairTerms r = pair_terms(q, p, all, count, inverse_weight(q, k, x[4]));
        if (threadIdx.x == 0) {
            q.ratios[2 * p] = (float)r.ratio[0];
            q.ratios[2 * p + 1] = (float)r.ratio[1];
            for (int j = 0; j < kTerms; ++j) k.terms[p * kTerms + j] = r.t[j];
            factors[0] = r.c[0];
            factors[1] = r.c[1];
        }
    }
    __syncthreads();
    c[0] = factors[0];
    c[1] = factors[1];
}

// ---------------------------------------------------------------------------
// heads of up to 64 actions
// ---------------------------------------------------------------------------

// A row in a group of G lanes, E actions each.
template <class T, int G, int E>
struct SmallRow {
    float x[E];          // logits, then exponentials
    float top, inverse;  // of the row
    float logp, ref;
    int at;              // the action, -1 where its probability is zero
    bool counts;

    __device__ __forceinline__ void read(const Rows& R, const Pairs& q, int64_t n, int member)
    {
        const int A = R.actions, i0 = member * E;
        const T* data = (const T*)R.data + n * R.stride;
        const uint8_t* mask = R.mask ? R.mask + n * R.mask_stride : nullptr;
        const int64_t action = q.actions[n];   // (no load waits for it)
        ref = q.ref ? q.ref[n] : 0.0f;
        T t[E];
        uint8_t m[E];
        const T* from = data + i0;
#pragma unroll
        for (int k = 0; k < E; k += 4) {
            if (i0 + k + 4 <= A) {
                __builtin_memcpy(t + k, from + k, 4 * sizeof(T));
                if (mask) __builtin_memcpy(m + k, mask + i0 + k, 4);
            } else {
#pragma unroll
                for (int j = k; j < k + 4; ++j) {
                    t[j] = (T)-INFINITY;
                    m[j] = 1;
                    if (i0 + j < A) {
                        t[j] = from[j];
                        if (mask) m[j] = mask[i0 + j];
                    }
                }
            }
        }
        float largest = -INFINITY, taken = -INFINITY;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            x[j] = mask && !m[j] ? -INFINITY : (float)t[j];
            largest = fmaxf(largest, x[j]);
            taken = i0 + j == action ? x[j] : taken;
        }
        counts = action >= 0 && action < A;
        at = counts ? (int)action : -1;
        logp = inverse = 0.0f;
        if (!counts) return;   // (the whole group)
        top = group_max<G>(largest);
        if constexpr (G > 1) taken = __shfl(taken, (threadIdx.x & 63 & ~(G - 1)) + at / E);
        const float base = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            x[j] = weight_of<T>(x[j], base);
            sum += x[j];
        }
        sum = group_sum<G>(sum);
        if (sum == 0.0f) {   // nothing is allowed
            counts = false;
            return;
        }
        inverse = 1.0f / sum;
        logp = (taken - base) - logf(sum);
        if (logp == -INFINITY) at = -1;
    }

    // c (delta - p), 0 at actions of probability zero
    __device__ __forceinline__ void write(const Rows& R, const Pairs& q, int64_t n, int member, float c) const
    {
        const int A = R.actions, i0 = member * E;
        T* out = (T*)q.dlogits + n * q.dstride + i0;
        const float f = counts ? -c * inverse : 0.0f;
        T t[E];
#pragma unroll
        for (int j = 0; j < E; ++j) t[j] = (T)(counts ? fmaf(f, x[j], i0 + j == at ? c : 0.0f) : 0.0f);
#pragma unroll
        for (int k = 0; k < E; k += 4) {
            if (i0 + k + 4 <= A) {
                __builtin_memcpy(out + k, t + k, 4 * sizeof(T));
            } else {
#pragma unroll
                for (int j = k; j < k + 4; ++j)
                    if (i0 + j < A) out[j] = t[j];
            }
        }
    }
};

constexpr int kOutside = 64;   // workgroups that clear the gradient of rows outside all sequences

// A workgroup to a pair.
template <class T, int G, int E>
__global__ __launch_bounds__(256) void pair_kernel(const Rows R, const Pairs q, const Scratch k)
{
    constexpr int kRows = 256 / G;   // of a workgroup at a time
    const int member = threadIdx.x % G, mine = threadIdx.x / G;
    SmallRow<T, G, E> row;
    if ((int64_t)blockIdx.x >= q.count) {
        const int64_t from = bound_of(q, 0, R.rows), to = bound_of(q, 2 * q.count, R.rows);
        row.counts = false;
        for (int64_t n = ((int64_t)blockIdx.x - q.count) * kRows + mine; n < R.rows; n += kOutside * kRows)
            if (n < from || n >= to) row.write(R, q, n, member, 0.0f);
        return;
    }
    const int64_t p = blockIdx.x;
    const int64_t first = bound_of(q, 2 * p, R.rows), middle = max(first, bound_of(q, 2 * p + 1, R.rows)),
                  last = max(middle, bound_of(q, 2 * p + 2, R.rows));
    double sum[2] = {};
    uint32_t rows[2] = {};
    for (int64_t n = first + mine; n < last; n += kRows) {
        row.read(R, q, n, member);
        if (row.counts && member == 0) {
            const double d = (double)(row.logp - row.ref);
            if (n < middle) sum[0] += d, ++rows[0];
            else sum[1] += d, ++rows[1];
        }
    }
    float factors[2];
    finish_pair(q, k, p, sum, rows, factors);
    const bool again = last - first > kRows;
    for (int64_t n = first + mine; n < last; n += kRows) {
        if (again) row.read(R, q, n, member);
        const float c = factors[n < middle ? 0 : 1];
        if (c == 0.0f) row.counts = false;   // (a pair of weight 0 may hold what is no number)
        row.write(R, q, n, member, c);
    }
}

// Sequences too long for a workgroup to a pair: every row's log-probability, ...
template <class T, int G, int E>
__global__ __launch_bounds__(256) void small_row_kernel(const Rows R, const Pairs q, const Scratch k)
{
    constexpr int kRows = 256 / G;
    const int member = threadIdx.x % G, mine = threadIdx.x / G;
    const int64_t from = bound_of(q, 0, R.rows), to = bound_of(q, 2 * q.count, R.rows);
    SmallRow<T, G, E> row;
    for (int64_t n = (int64_t)blockIdx.x * kRows + mine; n < R.rows; n += (int64_t)gridDim.x * kRows) {
        row.read(R, q, n, member);
        const bool on = row.counts && n >= from && n < to;
        if (member == 0) {
            k.factor[n] = on ? 1.0f : 0.0f;
            k.ratio[n] = on ? row.logp - row.ref : 0.0f;
        }
    }
}

// ... and, after terms_kernel, its gradient.
template <class T, int G, int E>
__global__ __launch_bounds__(256) void small_gradient_kernel(const Rows R, const Pairs q, const Scratch k)
{
    constexpr int kRows = 256 / G;
    const int member = threadIdx.x % G, mine = threadIdx.x / G;
    SmallRow<T, G, E> row;
    for (int64_t n = (int64_t)blockIdx.x * kRows + mine; n < R.rows; n += (int64_t)gridDim.x * kRows) {
        const float c = k.factor[n];
        row.read(R, q, n, member);
        if (c == 0.0f) row.counts = false;
        row.write(R, q, n, member, c);
    }
}

// ---------------------------------------------------------------------------
// larger heads
// ---------------------------------------------------------------------------

// V elements of a row from i on, -inf where nothing is allowed.
template <class T, int V>
struct Piece {
    T t[V];
    uint8_t m[V];
    __device__ __forceinline__ void load(const T* data, const uint8_t* mask, int i)
    {
        __builtin_memcpy(t, data + i, sizeof(t));
        if (mask) __builtin_memcpy(m, mask + i, sizeof(m));
    }
    __device__ __forceinline__ float operator()(const uint8_t* mask, int v) const { return mask && !m[v] ? -INFINITY : (float)t[v]; }
};

// The L lanes that work on a row: 16 (four rows a wave), a wave, or a workgroup of waves.
template <int L>
struct Team {
    static constexpr int kThreads = L < 256 ? 256 : L, kTeams = kThreads / L, kWaves = L < 64 ? 1 : L / 64;
    static constexpr int kInWave = L < 64 ? L : 64;
    __device__ __forceinline__ static int member() { return threadIdx.x % L; }
    __device__ __forceinline__ static int team() { return threadIdx.x / L; }
};

// Largest logit and sum of exponentials of every row, read once in vectors of 16 bytes at
// any address; the last one begins earlier where a row's length is no multiple of them, and
// its first elements are skipped.
template <class T, int L>
__global__ __launch_bounds__(Team<L>::kThreads) void row_kernel(const Rows R, const Pairs q, const Scratch k)
{
    using Tm = Team<L>;
    constexpr int V = 16 / sizeof(T), kAhead = 4, kTeams = Tm::kTeams, NW = Tm::kWaves;
    __shared__ float maxima[NW], sums[NW];
    const int member = Tm::member(), team = Tm::team();
    const int A = R.actions;
    const int64_t from = bound_of(q, 0, R.rows), to = bound_of(q, 2 * q.count, R.rows);
    for (int64_t n = (int64_t)blockIdx.x * kTeams + team; n < R.rows; n += (int64_t)gridDim.x * kTeams) {
        const int64_t action = q.actions[n];
        const bool on = action >= 0 && action < A && n >= from && n < to;
        if (!on) {   // (the whole team)
            if (member == 0) {
                k.factor[n] = 0.0f;
                k.ratio[n] = 0.0f;
            }
            continue;
        }
        const T* data = (const T*)R.data + n * R.stride;
        const uint8_t* mask = R.mask ? R.mask + n * R.mask_stride : nullptr;
        float top = -INFINITY, sum = 0.0f;
        auto add = [&](int i, auto whole) {   // whole: all of the vectors stand in the row
            constexpr bool kWhole = decltype(whole)::value;
            Piece<T, V> x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int at = i + u * L * V;
                if (kWhole || at < A) x[u].load(data, mask, kWhole || at + V <= A ? at : A - V);
            }
            float largest = -INFINITY;
            float y[kAhead][V];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int at = i + u * L * V, skip = at + V <= A ? 0 : at + V - A;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    y[u][v] = kWhole || (at < A && v >= skip) ? x[u](mask, v) : -INFINITY;
                    largest = fmaxf(largest, y[u][v]);
                }
            }
            if (largest > top) {
                sum *= weight_of<T>(top, largest);
                top = largest;
            }
            const float base = top == -INFINITY ? 0.0f : top;
            float some = 0.0f;
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int v = 0; v < V; ++v) some += weight_of<T>(y[u][v], base);
            sum += some;
        };
        constexpr int kChunk = L * V * kAhead;
        int i = member * V;
        for (; i - member * V + kChunk <= A; i += kChunk) add(i, Int<true>{});
        if (i < A) add(i, Int<false>{});
        float all = group_max<Tm::kInWave>(top);
        if constexpr (NW > 1) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) maxima[threadIdx.x >> 6] = all;
            __syncthreads();
            all = group_max<NW>(maxima[threadIdx.x & (NW - 1)]);
        }
        const float base = all == -INFINITY ? 0.0f : all;
        if (top != all) sum *= weight_of<T>(top, base);
        sum = group_sum<Tm::kInWave>(sum);
        if constexpr (NW > 1) {
            if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
            __syncthreads();
            sum = group_sum<NW>(sums[threadIdx.x & (NW - 1)]);
        }
        if (member == 0) {
            const float taken = mask && !mask[action] ? -INFINITY : (float)data[action];
            k.softmax[n] = make_float2(base, 1.0f / sum);
            k.factor[n] = sum == 0.0f ? 0.0f : 1.0f;   // nothing is allowed
            k.ratio[n] = sum == 0.0f ? 0.0f : (taken - base) - logf(sum) - (q.ref ? q.ref[n] : 0.0f);
        }
    }
}

// A workgroup to a pair: its sums, and the factors of its rows.
static __global__ __launch_bounds__(kPairThreads) void terms_kernel(const Pairs q, const Scratch k, int64_t all)
{
    constexpr int kAhead = 4;   // loads under way
    for (int64_t p = blockIdx.x; p < q.count; p += gridDim.x) {
        const int64_t first = bound_of(q, 2 * p, all), middle = max(first, bound_of(q, 2 * p + 1, all)),
                      last = max(middle, bound_of(q, 2 * p + 2, all));
        double sum[2] = {};
        uint32_t rows[2] = {};
        for (int64_t n = first + threadIdx.x; n < last; n += kAhead * kPairThreads) {
            float f[kAhead], d[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t i = n + u * kPairThreads;
                f[u] = i < last ? k.factor[i] : 0.0f;
                d[u] = i < last ? k.ratio[i] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const bool other = n + u * kPairThreads >= middle;
                sum[0] += other ? 0.0 : (double)d[u];
                sum[1] += other ? (double)d[u] : 0.0;
                rows[0] += !other && f[u] != 0.0f;
                rows[1] += other && f[u] != 0.0f;
            }
        }
        float c[2];
        finish_pair(q, k, p, sum, rows, c);
        for (int64_t n = first + threadIdx.x; n < last; n += kPairThreads)
            if (k.factor[n] != 0.0f) k.factor[n] = c[n < middle ? 0 : 1];
    }
}

// c (delta - p) of every row, by teams as in row_kernel; the first workgroup writes the
// statistics too.
template <class T, int L>
__global__ __launch_bounds__(Team<L>::kThreads) void gradient_kernel(const Rows R, const Pairs q, const Scratch k)
{
    using Tm = Team<L>;
    constexpr int V = 16 / sizeof(T), kTeams = Tm::kTeams;
    if (blockIdx.x == 0) write_stats<Tm::kThreads>(q, k);
    const int member = Tm::member(), team = Tm::team();
    const int A = R.actions;
    for (int64_t n = (int64_t)blockIdx.x * kTeams + team; n < R.rows; n += (int64_t)gridDim.x * kTeams) {
        const T* data = (const T*)R.data + n * R.stride;
        const uint8_t* mask = R.mask ? R.mask + n * R.mask_stride : nullptr;
        T* out = (T*)q.dlogits + n * q.dstride;
        const float c = k.factor[n];
        const bool on = c != 0.0f;
        const float2 s = on ? k.softmax[n] : make_float2(0.0f, 0.0f);
        const float f = -c * s.y;
        int action = -1;
        if (on) {
            action = (int)q.actions[n];
            if ((mask && !mask[action]) || (float)data[action] == -INFINITY) action = -1;
        }
        for (int i = member * V; i < A; i += L * V) {
            const int at = i + V <= A ? i : A - V;
            Piece<T, V> x;
            T y[V];
            if (on) x.load(data, mask, at);
#pragma unroll
            for (int v = 0; v < V; ++v) y[v] = (T)(on ? fmaf(f, weight_of<T>(x(mask, v), s.x), at + v == action ? c : 0.0f) : 0.0f);
            __builtin_memcpy(out + at, y, sizeof(y));
        }
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

constexpr int kSmallHead = 64;
// Rows of a pair, on average, from which on its sequences are spread over workgroups: two
// pairs of 4,096 rows of 12 take 43 us by a workgroup each and 20 spread, four of 2,000 rows
// 24 by a workgroup each.
// (The host knows no lengths but this mean: among 1,024 pairs one of 4,096 rows, 65,536 or a million
// takes 48 us, 669 or 10.6 ms, a pair of so many alone 22, 158 and 2.8 ms.)
constexpr int64_t kLongPair = 1024;

bool by_pairs(int64_t rows, int32_t actions, int64_t pairs) { return actions <= kSmallHead && rows <= kLongPair * pairs; }

uint64_t rounded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

uint64_t scratch_bytes(int64_t rows, int32_t actions, int64_t pairs)
{
    return 256 + rounded(pairs * kTerms * sizeof(double)) + (by_pairs(rows, actions, pairs) ? 0 : rounded(rows * 8) + 2 * rounded(rows * 4));
}

Scratch scratch_of(void* workspace, int64_t rows, int64_t pairs)
{
    char* at = (char*)workspace;
    Scratch k;
    k.omega = (double*)at;
    k.terms = (double*)(at += 256);
    k.softmax = (float2*)(at += rounded(pairs * kTerms * sizeof(double)));
    k.ratio = (float*)(at += rounded(rows * 8));
    k.factor = (float*)(at += rounded(rows * 4));
    return k;
}

template <class T>
void launch(const Rows& R, const Pairs& q, const Scratch& k, hipStream_t st)
{
    if (q.weights && q.denominator == 0.0f && q.count > kFewPairs)
        hipLaunchKernelGGL(weight_sum_kernel, dim3(1), dim3(1024), 0, st, q, k);
    auto with_rows = [&](auto go) {   // lanes of a row, elements of a lane
        if (R.actions <= 4) go(Int<1>{}, Int<4>{});
        else if (R.actions <= 8) go(Int<1>{}, Int<8>{});
        else if (R.actions <= 12) go(Int<1>{}, Int<12>{});
        else if (R.actions <= 16) go(Int<1>{}, Int<16>{});
        else go(Int<8>{}, Int<8>{});
    };
    auto terms = [&] {
        if (q.count > 0) hipLaunchKernelGGL(terms_kernel, dim3((unsigned)q.count), dim3(kPairThreads), 0, st, q, k, R.rows);
    };
    if (by_pairs(R.rows, R.actions, q.count)) {
        const dim3 grid((unsigned)(q.count + kOutside));
        with_rows([&](auto g, auto e) {
            hipLaunchKernelGGL((pair_kernel<T, decltype(g)::value, decltype(e)::value>), grid, dim3(256), 0, st, R, q, k);
        });
        hipLaunchKernelGGL(stats_kernel, dim3(1), dim3(256), 0, st, q, k);
        return;
    }
    if (R.actions <= kSmallHead) {
        with_rows([&](auto g, auto e) {
            constexpr int G = decltype(g)::value, E = decltype(e)::value;
            const int64_t all = (R.rows * G + 255) / 256, most = 1 << 20;
            const dim3 grid((unsigned)(all < most ? all : most));
            hipLaunchKernelGGL((small_row_kernel<T, G, E>), grid, dim3(256), 0, st, R, q, k);
            terms();
            hipLaunchKernelGGL((small_gradient_kernel<T, G, E>), grid, dim3(256), 0, st, R, q, k);
        });
        hipLaunchKernelGGL(stats_kernel, dim3(1), dim3(256), 0, st, q, k);
        return;
    }
    constexpr int V = 16 / sizeof(T);
    const int64_t vectors = (R.actions + V - 1) / V;
    auto go = [&](auto lanes) {
        using Tm = Team<decltype(lanes)::value>;
        constexpr int L = decltype(lanes)::value;
        const int64_t all = (R.rows + Tm::kTeams - 1) / Tm::kTeams, most = 1 << 20;
        const dim3 grid((unsigned)(all < 1 ? 1 : all < most ? all : most)), block(Tm::kThreads);
        hipLaunchKernelGGL((row_kernel<T, L>), grid, block, 0, st, R, q, k);
        terms();
        hipLaunchKernelGGL((gradient_kernel<T, L>), grid, block, 0, st, R, q, k);
    };
    if (vectors <= 96) go(Int<16>{});
    else if (vectors <= 512) go(Int<64>{});
    else if (vectors <= 4096) go(Int<256>{});
    else go(Int<1024>{});
}

constexpr int64_t kMostPairs = 1 << 23;   // (a launch has fewer than 2^32 threads)

pictura_status launched() { return hipGetLastError() == hipSuccess ? PICTURA_OK : PICTURA_EDEVICE; }

}  // namespace
}  // namespace pictura

using namespace pictura;

extern "C" {

pictura_status pictura_preference_loss_workspace(int64_t rows, int32_t actions, int64_t pairs, uint64_t* bytes)
{
    if (!bytes || rows < 0 || rows > 0x7FFFFFFFll || actions < 1 || actions > PICTURA_MAX_ACTIONS || pairs < 0 || pairs > kMostPairs)
        return PICTURA_EINVAL;
    *bytes = scratch_bytes(rows, actions, pairs);
    return PICTURA_OK;
}

pictura_status pictura_preference_loss(const pictura_logits* logits, const pictura_preferences* p, void* workspace,
                                       uint64_t workspace_bytes, float* out_stats, float* out_ratios, void* dlogits,
                                       int64_t dlogits_stride, void* stream)
{
    if (!logits_ok(logits) || !p || p->pairs < 0 || p->pairs > kMostPairs || !out_stats || !aligned(out_stats, 4)) return PICTURA_EINVAL;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < scratch_bytes(logits->rows, logits->actions, p->pairs))
        return PICTURA_EINVAL;
    if (!(p->beta > 0.0f) || !std::isfinite(p->beta) || !(p->smoothing >= 0.0f && p->smoothing < 1.0f) || !(p->denominator >= 0.0f) ||
        !std::isfinite(p->denominator))
        return PICTURA_EINVAL;
    if (!p->offsets || !aligned(p->offsets, 8) || !aligned(p->ref_logp, 4) || !aligned(p->weights, 4)) return PICTURA_EINVAL;
    if (p->pairs > 0 && (!out_ratios || !aligned(out_ratios, 4))) return PICTURA_EINVAL;
    if (logits->rows > 0) {
        if (!p->actions || !aligned(p->actions, 8) || !dlogits || !aligned(dlogits, size_of(logits->dtype))) return PICTURA_EINVAL;
        if (dlogits_stride < logits->actions && logits->rows > 1) return PICTURA_EINVAL;
    }
    const Rows R = rows_of(*logits);
    const Pairs q{p->actions, p->offsets, p->ref_logp, p->weights, p->pairs, p->beta, p->smoothing, p->denominator,
                  p->average ? 1 : 0, out_stats, out_ratios, dlogits, dlogits_stride};
    const Scratch k = scratch_of(workspace, R.rows, p->pairs);
    hipStream_t st = (hipStream_t)stream;
    if (logits->dtype == PICTURA_F32) launch<float>(R, q, k, st);
    else if (logits->dtype == PICTURA_BF16) launch<__bf16>(R, q, k, st);
    else launch<_Float16>(R, q, k, st);
    return launched();
}

}  // extern "C"
