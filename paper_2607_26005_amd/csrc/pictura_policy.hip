// The policy's decisions: actions drawn from logits, and the clipped policy loss
// over them with its gradient.
//
// Drawing.  The probabilities of a row are held as whole numbers, w = rint(2^31
// exp((x - max) / T)): sums of them are exact, so a draw does not depend on the order
// or the split of a sum, and a row draws alike alone and in any batch.  Weights below
// 2^-32 of the largest vanish.  What is kept by top_k and top_p is a prefix in the
// order of the logits, so a row needs the logit that the prefix ends with and not a
// sort.
//
// Both work on rows from a few actions to 2^20.  Up to 16 (loss) or 64 (drawing)
// actions a row takes a thread or a group of lanes; up to 73,728 it is held in the
// registers of one to sixteen waves and read once; longer ones are read again for
// every pass.
//
// Measured (a whole call among others; one MI355X, whose large copies run at 4,906
// GB/s and whose launches take 3.8 us): 65,536 rows of 12 drawn in 11.8 us, one row
// of 16,385 with top_k and top_p 10.4 us, 2,048 rows of 4,099 in bf16 with all three
// filters 30 us, 512 rows of 65,536 with top_p 96 us (134 MB read: 27 us at a copy's
// rate), without it 52 us; loss and gradient of 65,536 rows of 12 20.4 us, of 2,047
// rows of 16,381 in bf16 53 us (134 MB read and written).
#include <cmath>
#include <type_traits>

#include "pictura.h"
#include "pictura_policy.h"

#pragma clang fp contract(off)

namespace pictura {

// This file is compiled once for each type of logits, PICTURA_POLICY_TYPE, for the
// kernels, and once without for the entries.
#ifdef PICTURA_POLICY_TYPE

constexpr float kOne = 0x1p31f;           // weight of a row's largest logit
constexpr int kMaxBlocks = 1 << 20;       // workgroups of a launch, which then take rows in turn

// One row as the kernels read it: fp32, -inf at a place that is not allowed.
template <class T>
struct Row {
    const T* x;
    const uint8_t* mask;
    __device__ __forceinline__ Row(const Rows& r, int64_t n)
        : x((const T*)r.data + n * r.stride), mask(r.mask ? r.mask + n * r.mask_stride : nullptr) {}
    __device__ __forceinline__ float operator()(int i) const
    {
        return mask && !mask[i] ? -INFINITY : (float)x[i];
    }
};

// Bits in the order of the values (both zeros alike).
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// Weight of a logit against the row's largest.  The quotient (x - top) / T is the
// correctly rounded one, by a reciprocal and two corrections: with y = 1 / T rounded, q0 =
// d y is within two units of d / T, q1 = q0 + (d - q0 T) y within one, and from there
// one more step rounds correctly (Markstein, "Computation of elementary functions on
// the IBM RISC System/6000 processor", 1990).  Powers of two keep T and d where nothing
// underflows that could show, and quotients below -200 (an exponential of zero) are
// cut there, so that -inf gives weight 0.  At T = +inf every finite difference has the
// quotient 0: scale is 0 then, and -inf times 0 a NaN, which fmaxf drops for `least`.
struct Weights {
    float top, scale, temp, y, least;
    __device__ __forceinline__ Weights(float top_, float t) : top(top_)
    {
        scale = t < 0x1p-64f ? 0x1p100f : t > 0x1p64f ? t == INFINITY ? 0.0f : 0x1p-64f : 1.0f;
        temp = t == INFINITY ? 1.0f : t * scale;
        y = 1.0f / temp;
        least = -200.0f * temp;
    }
    __device__ __forceinline__ uint32_t operator()(float x) const
    {
        const float d = fmaxf((x - top) * scale, least);
        float q = d * y;
        q = fmaf(fmaf(-q, temp, d), y, q);
        q = fmaf(fmaf(-q, temp, d), y, q);
        return (uint32_t)rintf(expf(q) * kOne);
    }
};

// floor(total * m / 2^31) for m < 2^31
__device__ __forceinline__ uint64_t share(uint64_t total, uint32_t m)
{
    return (total >> 32) * m * 2 + ((total & 0xFFFFFFFFull) * m >> 31);
}

// floor(2^31 x) of x cut to [0, 1)
__device__ __forceinline__ uint32_t cut31(float x)
{
    return (uint32_t)(fminf(fmaxf(x, 0.0f), 1.0f - 0x1p-24f) * kOne);
}

// Lanes exchange through the vector unit's own data paths (row shifts and
// broadcasts): some 60 cycles for a reduction over the wave, where six shuffles
// through LDS take ten times that.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t lanes(uint32_t old, uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, kCtrl, kRows, 0xf, false);
}

template <int kCtrl, int kRows>
__device__ __forceinline__ uint64_t lanes(uint64_t old, uint64_t x)
{
    return (uint64_t)lanes<kCtrl, kRows>((uint32_t)(old >> 32), (uint32_t)(x >> 32)) << 32 |
           lanes<kCtrl, kRows>((uint32_t)old, (uint32_t)x);
}

template <int kCtrl, int kRows>
__device__ __forceinline__ double lanes(double old, double x)
{
    return __longlong_as_double((long long)lanes<kCtrl, kRows>((uint64_t)__double_as_longlong(old),
                                                               (uint64_t)__double_as_longlong(x)));
}

template <int kCtrl, int kRows>
__device__ __forceinline__ float lanes(float old, float x)
{
    return __uint_as_float(lanes<kCtrl, kRows>(__float_as_uint(old), __float_as_uint(x)));
}

// x of this lane combined with those before it: within 16 lanes (L = 16), or
// over the wave (L = 64).  `none` is what lanes that do not exist hold.
template <int L, class V, class F>
__device__ __forceinline__ V lane_scan(V x, V none, F f)
{
    x = f(x, lanes<0x111, 0xf>(none, x));
    if constexpr (L > 2) x = f(x, lanes<0x112, 0xf>(none, x));
    if constexpr (L > 4) x = f(x, lanes<0x114, 0xf>(none, x));
    if constexpr (L > 8) x = f(x, lanes<0x118, 0xf>(none, x));
    if constexpr (L > 16) x = f(x, lanes<0x142, 0xa>(none, x));
    if constexpr (L > 32) x = f(x, lanes<0x143, 0xc>(none, x));
    return x;
}

__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane)
{
    return (uint64_t)from_lane((uint32_t)(x >> 32), lane) << 32 | from_lane((uint32_t)x, lane);
}

__device__ __forceinline__ double from_lane(double x, int lane)
{
    return __longlong_as_double((long long)from_lane((uint64_t)__double_as_longlong(x), lane));
}

__device__ __forceinline__ float from_lane(float x, int lane) { return __uint_as_float(from_lane(__float_as_uint(x), lane)); }

struct Add {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// Running sum over the wave's lanes, this one included; and the whole sum or maximum.
template <class V>
__device__ __forceinline__ V wave_scan(V x) { return lane_scan<64>(x, (V)0, Add{}); }

template <class V>
__device__ __forceinline__ V wave_sum(V x) { return from_lane(wave_scan(x), 63); }

__device__ __forceinline__ float wave_max(float x) { return from_lane(lane_scan<64>(x, -INFINITY, Max{}), 63); }

// Sum or maximum over a workgroup of NW waves, the same in every thread.  lds[NW]
// must not be in use by the threads before this call's barrier: two calls in a
// row take two arrays.
template <int NW, class V>
__device__ __forceinline__ V block_sum(V x, V* lds)
{
    x = wave_sum(x);
    if constexpr (NW == 1) return x;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return from_lane(lane_scan<NW>(lds[threadIdx.x & (NW - 1)], (V)0, Add{}), NW - 1);
}

template <int NW>
__device__ __forceinline__ float block_max(float x, float* lds)
{
    x = wave_max(x);
    if constexpr (NW == 1) return x;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return from_lane(lane_scan<NW>(lds[threadIdx.x & (NW - 1)], -INFINITY, Max{}), NW - 1);
}

// A prefix of the actions ordered by logit, then index: everything above `key`
// and the first `ties` of those with it.
struct Cut {
    uint32_t key;
    uint32_t ties;
};

// Histogram of whole numbers, its bins padded apart so that a lane can walk
// through consecutive ones.
__device__ __forceinline__ int padded(int bin) { return bin + (bin >> 4); }

// First bin of `bins` (a multiple of 64, at most 4096) up to which the sums reach
// need, by one wave; told = {bin, need less the bins before it}.  need is at most the
// sum of all.
template <class H>
__device__ __forceinline__ void find_bin(const H* hist, int bins, uint64_t need, uint64_t* told)
{
    const int lane = threadIdx.x & 63, per = bins / 64;
    uint64_t mine = 0;
    for (int i = 0; i < per; ++i) mine += hist[padded(lane * per + i)];
    uint64_t run = wave_scan(mine);
    const int at = __ffsll((unsigned long long)__ballot(run >= need)) - 1;
    need -= from_lane(run - mine, at);
    mine = lane < per ? hist[padded(at * per + lane)] : 0;   // that lane's bins, one each
    run = wave_scan(mine);
    const int in = __ffsll((unsigned long long)__ballot(run >= need)) - 1;
    if (lane == in) {
        told[0] = (uint64_t)(at * per + in);
        told[1] = need - (run - mine);
    }
}

// Smallest count of weights `one` that reaches `need` (below 2^52, a quotient up
// to 2^20): exact in fp64.
__device__ __forceinline__ uint32_t ties_for(uint64_t need, uint64_t one)
{
    return (uint32_t)ceil((double)need / (double)one);
}

// The shortest prefix whose sum of add(x) reaches `need` > 0, of the logits above
// floor_key that each(f) hands to f, spread over the threads; need is at most the
// sum of all of those.  By bytes of the key, from the highest: a histogram of the
// sums, largest byte first, up to where need is reached.
template <class Each, class Add>
__device__ Cut find_cut(Each each, uint32_t floor_key, uint64_t need, Add add, unsigned long long* hist, uint64_t* told)
{
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < padded(256); i += blockDim.x) hist[i] = 0;
        __syncthreads();
        each([&](float x) {
            const uint32_t k = order_key(x);
            if (x == -INFINITY || k <= floor_key || (shift < 24 && (k >> (shift + 8)) != prefix)) return;
            atomicAdd(&hist[padded(255 - ((k >> shift) & 255u))], (unsigned long long)add(x));
        });
        __syncthreads();
        if (threadIdx.x < 64) find_bin(hist, 256, need, told);
        __syncthreads();
        prefix = prefix << 8 | (255u - (uint32_t)told[0]);
        need = told[1];
    }
    __syncthreads();
    return Cut{prefix, ties_for(need, add(key_value(prefix)))};
}

// x as a value that is the same in every lane, which the compiler then knows.
__device__ __forceinline__ uint32_t same_in_wave(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

__device__ __forceinline__ uint64_t same_in_wave(uint64_t x)
{
    return (uint64_t)same_in_wave((uint32_t)(x >> 32)) << 32 | same_in_wave((uint32_t)x);
}

__device__ __forceinline__ float same_in_wave(float x) { return __uint_as_float(same_in_wave(__float_as_uint(x))); }

// A row's settings.
struct RowSampling {
    float temp, top_p, u;
    int32_t top_k;
    uint32_t least;   // smallest weight that is kept
    bool greedy;
    __device__ __forceinline__ RowSampling(const Sampling& S, const float* uniform, int64_t n)
    {
        temp = same_in_wave(S.temperatures ? S.temperatures[n] : S.temperature);
        top_k = (int32_t)same_in_wave((uint32_t)(S.top_ks ? S.top_ks[n] : S.top_k));
        top_p = same_in_wave(S.top_ps ? S.top_ps[n] : S.top_p);
        const float min_p = same_in_wave(S.min_ps ? S.min_ps[n] : S.min_p);
        least = (uint32_t)ceilf(fminf(fmaxf(min_p, 0.0f), 1.0f) * kOne);
        u = same_in_wave(uniform[n]);
        // The first of the largest logits: at this temperature any smaller one weighs less
        // than 2^31 (the least difference, 2^-149, makes it 2^31 - 2^8), and 0 draws the first.
        greedy = temp == 0.0f;
        if (greedy) {
            temp = 0x1p-126f;
            least = 1u << 31;
            top_k = 0;
            top_p = 1.0f;
            u = 0.0f;
        }
    }
};

// ---------------------------------------------------------------------------
// rows of any length: read again for every pass
// ---------------------------------------------------------------------------

// Sixteen waves to a row, eight loads of each thread under way: bound by the loads'
// latency.  256 rows of 131,072 in fp32 are drawn in 80 us without filters and 221 with
// top_p (170 and 437 with one load at a time), their loss and gradient take 107 us (571
// with four waves and one load; bf16 100).  A row stays on one CU, however few rows
// there are: one of 131,072 with both filters takes 175 us.
constexpr int kLongWaves = 16;
constexpr int kAhead = 8;   // loads of a thread that are under way together

// The logits at i, i + step, ...  Masked ones are loaded too: no load waits for another.
template <class T>
__device__ __forceinline__ void load_ahead(const Row<T>& row, int i, int step, float (&x)[kAhead])
{
    T t[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) t[u] = row.x[i + u * step];
    if (row.mask) {
        uint8_t m[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) m[u] = row.mask[i + u * step];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u] = m[u] ? (float)t[u] : -INFINITY;
    } else {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u] = (float)t[u];
    }
}

// f(i, x) for the logits of a row at i0, i0 + step, ... below i1, in that order.
template <class T, class F>
__device__ __forceinline__ void walk_row(const Row<T>& row, int i0, int i1, int step, F f)
{
    int i = i0;
    for (; i < i1 - (kAhead - 1) * step; i += kAhead * step) {
        float x[kAhead];
        load_ahead(row, i, step, x);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) f(i + u * step, x[u]);
    }
    for (; i < i1; i += step) f(i, row(i));
}

template <class T>
__global__ __launch_bounds__(kLongWaves * 64) void sample_long_kernel(const Rows R, const Sampling S,
                                                                      const float* __restrict__ uniform,
                                                                      int64_t* __restrict__ out_action,
                                                                      float* __restrict__ out_logp)
{
    constexpr int NW = kLongWaves, NT = NW * 64;
    __shared__ unsigned long long hist[256 + 16];
    __shared__ uint64_t told[2], lds64[3 * NW];
    __shared__ float ldsf[2 * NW];
    __shared__ uint32_t wties[NW];
    const int A = R.actions;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t n = blockIdx.x; n < R.rows; n += gridDim.x) {
        const Row<T> row(R, n);
        const RowSampling q(S, uniform, n);
        auto each = [&](auto f) { walk_row(row, threadIdx.x, A, NT, [&](int, float x) { f(x); }); };
        // the largest logit; a NaN or +inf, or a temperature without meaning, makes no draw
        float top = -INFINITY, bad = q.temp >= 0.0f ? 0.0f : 1.0f;
        each([&](float x) {
            top = fmaxf(top, x);
            if (!(x < INFINITY)) bad = 1.0f;
        });
        top = block_max<NW>(top, ldsf);
        bad = block_max<NW>(bad, ldsf + NW);
        if (bad != 0.0f || top == -INFINITY) {
            if (threadIdx.x == 0) {
                out_action[n] = -1;
                out_logp[n] = NAN;
            }
            __syncthreads();
            continue;
        }
        const Weights weight(top, q.temp);
        Cut cut{0u, 0u};
        if (q.top_k > 0 && q.top_k < A) {
            uint64_t some = 0;
            each([&](float x) { some += x != -INFINITY; });
            if (block_sum<NW>(some, lds64) > (uint64_t)q.top_k)
                cut = find_cut(each, 0u, (uint64_t)q.top_k, [](float) { return 1u; }, hist, told);
        }
        if (q.top_p < 1.0f) {
            uint64_t above = 0;
            each([&](float x) {
                if (order_key(x) > cut.key) above += weight(x);
            });
            above = block_sum<NW>(above, lds64 + NW);
            const uint64_t one = cut.ties ? weight(key_value(cut.key)) : 0;
            uint64_t need = share(above + one * cut.ties, cut31(q.top_p));
            if (need < 1) need = 1;
            if (need <= above) cut = find_cut(each, cut.key, need, weight, hist, told);
            else cut.ties = ties_for(need - above, one);
        }
        auto kept = [&](float x) {
            const uint32_t w = weight(x);
            return w < q.least ? 0u : w;
        };
        // each wave its part of the row; the ties belong to the first waves that have them
        const int per = ((A + NT - 1) / NT) * 64, i0 = min(A, wave * per), i1 = min(A, i0 + per);
        uint64_t sum = 0;
        uint32_t ties = 0;
        walk_row(row, i0 + lane, i1, 64, [&](int, float x) {
            const uint32_t key = order_key(x);
            if (x == -INFINITY) return;
            if (key > cut.key) sum += kept(x);
            ties += key == cut.key;
        });
        sum = wave_sum(sum);
        ties = wave_sum(ties);
        const uint32_t one = cut.ties ? kept(key_value(cut.key)) : 0u;
        if (lane == 0) {
            lds64[2 * NW + wave] = sum;
            wties[wave] = ties;
        }
        __syncthreads();
        // where this wave's part of the running sum begins, and how many ties are left for it
        uint64_t total = 0, base = 0, mine = 0;
        uint32_t quota = cut.ties, left = 0;
        for (int w = 0; w < NW; ++w) {
            const uint32_t take = min(quota, wties[w]);
            const uint64_t part = lds64[2 * NW + w] + (uint64_t)take * one;
            if (w == wave) {
                base = total;
                mine = part;
                left = take;
            }
            quota -= take;
            total += part;
        }
        const uint64_t target = share(total, cut31(q.u));
        if (base <= target && target - base < mine) {   // one wave: it walks through its part
            for (int b = i0; b < i1; b += kAhead * 64) {
                float x[kAhead];
                uint32_t w[kAhead];
                uint64_t some = 0;
                if (b + kAhead * 64 <= i1) {
                    load_ahead(row, b + lane, 64, x);
                } else {
#pragma unroll
                    for (int v = 0; v < kAhead; ++v) {
                        const int i = b + v * 64 + lane;
                        x[v] = i < i1 ? row(i) : -INFINITY;
                    }
                }
#pragma unroll
                for (int v = 0; v < kAhead; ++v) {
                    const uint32_t key = order_key(x[v]);
                    const bool tie = x[v] != -INFINITY && key == cut.key;
                    const uint64_t same = __ballot(tie);
                    const uint32_t before = __popcll(same & ((1ull << lane) - 1ull));
                    w[v] = x[v] == -INFINITY ? 0u : key > cut.key || (tie && before < left) ? kept(x[v]) : 0u;
                    left -= min(left, (uint32_t)__popcll(same));
                    some += w[v];
                }
                some = wave_sum(some);
                if (base + some <= target) {
                    base += some;
                    continue;
                }
                bool found = false;
#pragma unroll
                for (int v = 0; v < kAhead; ++v) {
                    const uint64_t run = wave_scan((uint64_t)w[v]);
                    const uint64_t hit = __ballot(base + run > target);
                    if (hit && !found && lane == __ffsll((unsigned long long)hit) - 1) {
                        out_action[n] = b + v * 64 + lane;
                        out_logp[n] = q.greedy ? 0.0f : logf((float)w[v] / (float)total);
                    }
                    found = found || hit;
                    base += __shfl(run, 63);
                }
                break;
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// rows that fit a workgroup's registers
// ---------------------------------------------------------------------------

// Bits of a number up to 2^31 as a float, which keeps the order.
__device__ __forceinline__ uint32_t float_bits(uint32_t w) { return __float_as_uint((float)w); }

constexpr uint32_t kOneBits = 0x4F000000u;   // of 2^31

// Says that x may be new from here on: what was computed from it in an earlier pass
// over a thread's registers is not kept for this one (it would take as many
// registers again).
template <int V>
__device__ __forceinline__ void renew(uint32_t (&x)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) asm volatile("" : "+v"(x[v]));
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A row of V-element vectors at addresses that are a multiple of them: vector q covers the elements
// from q V - shift on, the first and the last perhaps only in part.  A thread of
// a workgroup of NW waves holds up to NV of them, 64 vectors apart, and a wave a
// stretch of the row.
template <class T, int NW, int NV, int V>
struct VecRow {
    Row<T> row;
    int A, shift, vectors, per, q0;
    __device__ __forceinline__ VecRow(const Rows& r, int64_t n, int wave, int lane) : row(r, n), A(r.actions)
    {
        shift = (int)(reinterpret_cast<uintptr_t>(row.x) / sizeof(T)) & (V - 1);
        vectors = (A + shift + V - 1) / V;
        per = (vectors + NW * 64 - 1) / (NW * 64);   // vectors of a thread, at most NV
        q0 = wave * per * 64 + lane;                 // its first one
    }
    __device__ __forceinline__ int first(int j) const { return (q0 + j * 64) * V - shift; }
    // whole vectors: q in [from, to)
    __device__ __forceinline__ int from() const { return shift ? 1 : 0; }
    __device__ __forceinline__ int to() const { return (A + shift) / V; }
    __device__ __forceinline__ bool whole(int j) const { return q0 + j * 64 >= from() && q0 + j * 64 < to(); }

    // The logits' bits, -inf where there is none.
    __device__ __forceinline__ void load(uint32_t (&r)[NV][V]) const
    {
        struct alignas(V * sizeof(T)) Vec { T v[V]; };
        const Vec* at = reinterpret_cast<const Vec*>(row.x - shift) + q0;
        const uint32_t none = __float_as_uint(-INFINITY);
        if constexpr (sizeof(T) == 2) {
            // All loads first, then the conversions (a conversion next to its load waits for
            // it before the next one leaves), four at a time as registers that belong
            // together: one by one the compiler keeps every logit twice.
            typedef uint32_t Words __attribute__((ext_vector_type(V / 2)));
            const uint32_t half = (uint32_t)__builtin_bit_cast(uint16_t, (T)-INFINITY) * 0x10001u;
            Words raw[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                raw[j] = (Words)half;
                if (j < per && whole(j)) raw[j] = reinterpret_cast<const Words*>(at)[j * 64];
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const Vec t = __builtin_bit_cast(Vec, raw[j]);
#pragma unroll
                for (int k = 0; k < V; k += 4) {
                    u32x4 y;
#pragma unroll
                    for (int v = 0; v < 4; ++v) y[v] = __float_as_uint((float)t.v[k + v]);
                    asm volatile("" : "+v"(y));
#pragma unroll
                    for (int v = 0; v < 4; ++v) r[j][k + v] = y[v];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int v = 0; v < V; ++v) r[j][v] = none;
                if (j < per && whole(j)) {
                    const Vec t = at[j * 64];
#pragma unroll
                    for (int v = 0; v < V; ++v) r[j][v] = __float_as_uint((float)t.v[v]);
                }
            }
        }
        // the two ends, element by element
        const int last = vectors - 1 - q0;
        const int je = last >= 0 && !(last & 63) && to() < vectors && (last >> 6) < per ? last >> 6 : -1;
        if (q0 == 0 && shift) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v >= shift && v - shift < A) r[0][v] = __float_as_uint((float)row.x[v - shift]);
        }
        if (je >= 0 && (je > 0 || q0 > 0 || !shift)) {
            uint32_t t[V];
            const int i0 = first(je);
#pragma unroll
            for (int v = 0; v < V; ++v) t[v] = i0 + v < A ? __float_as_uint((float)row.x[i0 + v]) : none;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) r[j][v] = j == je ? t[v] : r[j][v];
        }
        if (row.mask) {
            struct Bytes { uint8_t v[V]; };
            if constexpr (V == 4) {
                // four loads, at any address, before the first is waited for; more (and two
                // of eight) take registers of which the kernels have none left
                constexpr int kGroup = 4;
#pragma unroll
                for (int j0 = 0; j0 < NV; j0 += kGroup) {
                    uint32_t m[kGroup];
#pragma unroll
                    for (int g = 0; g < kGroup; ++g) {
                        const int j = j0 + g;
                        m[g] = 0x01010101u;
                        if (j < NV && j < per && whole(j)) __builtin_memcpy(&m[g], row.mask + first(j), V);
                    }
#pragma unroll
                    for (int g = 0; g < kGroup; ++g) {
                        const int j = j0 + g;
                        if (j < NV && j < per) {
                            const Bytes k = __builtin_bit_cast(Bytes, m[g]);
                            if (!whole(j)) mask_ends(j, r[j]);
#pragma unroll
                            for (int v = 0; v < V; ++v) r[j][v] = k.v[v] ? r[j][v] : none;
                        }
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (j < per) {
                        if (whole(j)) {
                            Bytes k;
                            __builtin_memcpy(&k, row.mask + first(j), V);
#pragma unroll
                            for (int v = 0; v < V; ++v) r[j][v] = k.v[v] ? r[j][v] : none;
                        } else {
                            mask_ends(j, r[j]);
                        }
                    }
            }
        }
    }
    // a vector that the row covers only in part
    __device__ __forceinline__ void mask_ends(int j, uint32_t (&x)[V]) const
    {
        const int i0 = first(j);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (i0 + v >= 0 && i0 + v < A && !row.mask[i0 + v]) x[v] = __float_as_uint(-INFINITY);
    }
};

constexpr int kMostSlots = 16 * 64 * 72;   // longest row that registers hold
constexpr int kRank = 256;   // candidates that are ranked by counting

// Shared memory of a row's workgroup.
template <int NW, bool kFilter>
struct RowLds {
    static constexpr int kBins = NW == 1 ? 256 : 1024, kList = NW == 1 ? 512 : 2048;
    alignas(16) unsigned long long hist[kFilter ? kBins + kBins / 16 : 1];
    alignas(16) float list[kFilter ? kList + 4 : 1];        // candidates
    alignas(16) uint32_t weight[kFilter ? kRank + 4 : 1];   // theirs
    alignas(16) int32_t index[kFilter ? kRank + 4 : 1];     // and where they stand
    uint64_t sums[2][NW], told[5];
    uint32_t listed;
    float maxima[3][NW];
    uint32_t ties[NW];
};

constexpr uint32_t kTie = 0xFFFFFFFFu;   // in a weight's place: equal to the cut

constexpr int kSmallBins = 256;

// First of kSmallBins bins up to which the counts reach need, the last where they do
// not; every wave for itself.
__device__ __forceinline__ int find_small_bin(const uint32_t* hist, uint32_t need)
{
    const int lane = threadIdx.x & 63;
    const uint4 h = *reinterpret_cast<const uint4*>(hist + 4 * lane);
    const uint32_t mine = h.x + h.y + h.z + h.w, run = wave_scan(mine);
    const uint64_t hit = __ballot(run >= need);
    if (!hit) return kSmallBins - 1;
    const int at = __ffsll((unsigned long long)hit) - 1;
    const uint32_t left = need - from_lane(run - mine, at);
    const uint32_t a = from_lane(h.x, at), b = from_lane(h.y, at), c = from_lane(h.z, at);
    return 4 * at + (left <= a ? 0 : left <= a + b ? 1 : left <= a + b + c ? 2 : 3);
}

// What one wave wrote to LDS is there for its other lanes.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
}

// The draw among C <= kRank candidates, which hold the top_k largest logits: each is
// ranked by counting those above it.  (A loop over four candidates at a time waits
// for LDS some 130 cycles: few candidates, and spread over the waves.)
template <int NW, class Lds>
__device__ __forceinline__ void draw_from_list(Lds& lds, uint32_t C, const Weights& weight, const RowSampling& q,
                                               int64_t n, int64_t* __restrict__ out_action, float* __restrict__ out_logp)
{
    constexpr uint32_t NT = NW * 64;
    constexpr int Q = kRank / NT < 1 ? 1 : kRank / NT;   // candidates of a thread
    const uint32_t k = min((uint32_t)q.top_k, C), wave0 = threadIdx.x & ~63u;
    const bool nucleus = q.top_p < 1.0f;
    float x[Q];
    uint32_t w[Q], above[Q], equal[Q];
    uint64_t before[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const uint32_t c = threadIdx.x + NT * i;
        x[i] = -INFINITY;
        w[i] = above[i] = equal[i] = 0;
        before[i] = 0;
        if (wave0 + NT * i < C) {
            if (c < C) x[i] = lds.list[c];
            w[i] = weight(x[i]);
            if (c < kRank) lds.weight[c] = w[i];   // (past C: 0)
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < Q; ++i)
        if (wave0 + NT * i < C) {
#pragma unroll 2
            for (uint32_t b = 0; b < C; b += 4) {   // (past C: -inf)
                const float4 y = *reinterpret_cast<const float4*>(lds.list + b);
                const uint4 z = *reinterpret_cast<const uint4*>(lds.weight + b);
                above[i] += (y.x > x[i]) + (y.y > x[i]) + (y.z > x[i]) + (y.w > x[i]);
                equal[i] += (y.x == x[i]) + (y.y == x[i]) + (y.z == x[i]) + (y.w == x[i]);
                before[i] += (uint64_t)(y.x > x[i] ? z.x : 0u) + (y.y > x[i] ? z.y : 0u);
                before[i] += (uint64_t)(y.z > x[i] ? z.z : 0u) + (y.w > x[i] ? z.w : 0u);
            }
            if (threadIdx.x + NT * i < C && above[i] < k && k <= above[i] + equal[i]) {   // (equal ones write the same)
                lds.told[0] = (uint64_t)equal[i] << 32 | __float_as_uint(x[i]);
                lds.told[1] = k - above[i];
                lds.told[2] = before[i] + (uint64_t)(k - above[i]) * w[i];
            }
        }
    __syncthreads();
    float over = __uint_as_float(same_in_wave((uint32_t)lds.told[0]));
    uint32_t same = same_in_wave((uint32_t)(lds.told[0] >> 32)), ties = same_in_wave((uint32_t)lds.told[1]);
    if (nucleus) {
        uint64_t need = share(lds.told[2], cut31(q.top_p));
        if (need < 1) need = 1;
#pragma unroll
        for (int i = 0; i < Q; ++i)
            if (threadIdx.x + NT * i < C && x[i] >= over) {
                const uint32_t some = x[i] == over ? ties : equal[i];
                if (before[i] < need && need <= before[i] + (uint64_t)some * w[i]) {
                    lds.told[3] = (uint64_t)equal[i] << 32 | __float_as_uint(x[i]);
                    lds.told[4] = ties_for(need - before[i], w[i]);
                }
            }
        __syncthreads();
        over = __uint_as_float(same_in_wave((uint32_t)lds.told[3]));
        same = same_in_wave((uint32_t)(lds.told[3] >> 32));
        ties = same_in_wave((uint32_t)lds.told[4]);
    }
    // what is left of each weight
    uint32_t index[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const uint32_t c = threadIdx.x + NT * i;
        index[i] = 0xFFFFFFFFu;
        if (wave0 + NT * i < C) {
            if (c < C) index[i] = (uint32_t)lds.index[c];
            bool in = c < C && x[i] >= over && w[i] >= q.least;
            if (ties < same && __any(in && x[i] == over)) {   // the first of the equal ones, by index
                uint32_t ahead = 0;
#pragma unroll 2
                for (uint32_t b = 0; b < C; b += 4) {
                    const float4 y = *reinterpret_cast<const float4*>(lds.list + b);
                    const int4 z = *reinterpret_cast<const int4*>(lds.index + b);
                    ahead += (y.x == x[i] && (uint32_t)z.x < index[i]) + (y.y == x[i] && (uint32_t)z.y < index[i]);
                    ahead += (y.z == x[i] && (uint32_t)z.z < index[i]) + (y.w == x[i] && (uint32_t)z.w < index[i]);
                }
                in = in && (x[i] > over || ahead < ties);
            }
            w[i] = in ? w[i] : 0u;
            if (c < kRank) lds.weight[c] = w[i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < Q; ++i)
        if (__any(w[i] != 0)) {
            uint64_t total = 0, first = 0;   // all weights, and those that come before by index
#pragma unroll 2
            for (uint32_t b = 0; b < C; b += 4) {
                const int4 y = *reinterpret_cast<const int4*>(lds.index + b);
                const uint4 z = *reinterpret_cast<const uint4*>(lds.weight + b);
                total += (uint64_t)z.x + z.y;
                total += (uint64_t)z.z + z.w;
                first += (uint64_t)((uint32_t)y.x < index[i] ? z.x : 0u) + ((uint32_t)y.y < index[i] ? z.y : 0u);
                first += (uint64_t)((uint32_t)y.z < index[i] ? z.z : 0u) + ((uint32_t)y.w < index[i] ? z.w : 0u);
            }
            const uint64_t target = share(total, cut31(q.u));
            if (first <= target && target - first < w[i]) {
                out_action[n] = (int64_t)index[i];
                out_logp[n] = q.greedy ? 0.0f : logf((float)w[i] / (float)total);
            }
        }
}

// One workgroup of NW waves per row, ITEMS logits to a thread, read once.  Each
// wave holds a stretch of the row, 64 vectors at a time, so that running sums by
// index go wave by wave.  A cut is found (the value that the kept prefix ends
// with, and how many of the logits equal to it are kept), then the registers hold
// the weights that are left, then the draw goes by their sums.
//
// top_k needs no exponentials but its candidates': a histogram of the maxima of four
// bounds them from below, and most rows end with the few that are listed (2,048 rows
// of 4,099 in fp32: 25 us with top_k 64, with or without top_p 0.95, and 15 without
// filters).  top_p alone needs all weights, then a histogram by weight of those that
// can matter (30 us).
// 512 rows of 65,536 with top_p: 96 us, the vector unit issues in 63 % of it, 75
// instructions for 64 logits.  A CU's registers hold one such row, so no loads run
// under the arithmetic of another.
// In bf16 the same takes 89 us; 1,024 rows of 32,768 take 90 and 93 (fp32).
template <class T, int NW, int ITEMS, bool kFilter>
__global__ __launch_bounds__(NW * 64) void sample_row_kernel(const Rows R, const Sampling S,
                                                             const float* __restrict__ uniform,
                                                             int64_t* __restrict__ out_action,
                                                             float* __restrict__ out_logp)
{
    // (with a filter four elements to a vector, whatever their type: eight take more
    // registers)
    constexpr int V = kFilter ? 4 : 16 / sizeof(T), NV = ITEMS / V, NT = NW * 64;
    using Lds = RowLds<NW, kFilter>;
    __shared__ alignas(16) Lds lds;
    const int A = R.actions;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= R.rows) return;
    const VecRow<T, NW, NV, V> vr(R, n, wave, lane);
    const Row<T>& row = vr.row;
    const RowSampling q(S, uniform, n);
    const int per = vr.per;
    // bits of the logits, later the weights
    uint32_t r[NV][V];
    float top = -INFINITY;
    bool odd = !(q.temp >= 0.0f);
    vr.load(r);
    auto x = [&](int j, int v) { return __uint_as_float(r[j][v]); };
    auto vmax = [&](int j) {
        float m = x(j, 0);
#pragma unroll
        for (int v = 1; v < V; ++v) m = fmaxf(m, x(j, v));
        return m;
    };
    float low = INFINITY;   // smallest of the fours' maxima
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (j < per) {
            renew(r[j]);
            const float m = vmax(j);
            top = fmaxf(top, m);
            if (kFilter) low = m > -INFINITY ? fminf(low, m) : low;
#pragma unroll
            for (int v = 0; v < V; ++v) odd |= !(x(j, v) < INFINITY);
        }
    const bool some_k = kFilter && q.top_k > 0 && q.top_k < A;
    uint32_t* const counts = reinterpret_cast<uint32_t*>(lds.hist);
    if constexpr (kFilter) {
        if (some_k) {
            for (int i = threadIdx.x; i < kSmallBins; i += NT) counts[i] = 0;
            for (int i = threadIdx.x; i < kRank + 4; i += NT) lds.list[i] = -INFINITY;
        }
        if (threadIdx.x == 0) lds.listed = 0;
    }
    // the largest logit; a NaN or +inf, or a temperature without meaning, makes no draw
    top = wave_max(odd ? INFINITY : top);
    if (kFilter) low = -wave_max(-low);
    if constexpr (NW > 1) {
        if (lane == 0) {
            lds.maxima[0][wave] = top;
            lds.maxima[1][wave] = -low;
        }
        __syncthreads();
        top = from_lane(lane_scan<NW>(lds.maxima[0][lane & (NW - 1)], -INFINITY, Max{}), NW - 1);
        if (kFilter) low = -from_lane(lane_scan<NW>(lds.maxima[1][lane & (NW - 1)], -INFINITY, Max{}), NW - 1);
    } else if (kFilter) {
        wave_fence();
    }
    if (top == INFINITY || top == -INFINITY) {
        if (threadIdx.x == 0) {
            out_action[n] = -1;
            out_logp[n] = NAN;
        }
        return;
    }
    const Weights weight(top, q.temp);
    // The cut: logits over `over` are kept, and the first `ties` of those equal to it.
    float over = -INFINITY;
    uint32_t ties = 0;
    bool by_logit = false;   // the cut comes from the logits, before any weight
    if constexpr (kFilter) {
        if (some_k) {
            // The top_k-th largest of the maxima of four is no more than the top_k-th
            // largest logit: a histogram of them bounds the logits that can be kept
            // from below, and those few are listed.
            const float scale = (float)kSmallBins / (top - low);   // (no range: NaN, and all in bin 0)
            auto bin = [&](float y) { return (int)fminf(fmaxf((top - y) * scale, 0.0f), (float)(kSmallBins - 1)); };
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
                    const float m = vmax(j);
                    if (m > -INFINITY) atomicAdd(&counts[bin(m)], 1u);
                }
            __syncthreads();
            const int edge = find_small_bin(counts, (uint32_t)q.top_k);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
                    const float m = vmax(j);
                    if (m > -INFINITY && bin(m) <= edge) {
#pragma unroll
                        for (int v = 0; v < V; ++v)
                            if (x(j, v) > -INFINITY && bin(x(j, v)) <= edge) {
                                const uint32_t at = atomicAdd(&lds.listed, 1u);
                                if (at < Lds::kList) lds.list[at] = x(j, v);
                                if (at < kRank) lds.index[at] = vr.first(j) + v;
                            }
                    }
                }
            __syncthreads();
            const uint32_t C = same_in_wave(lds.listed);
            if (C <= kRank) {
                draw_from_list<NW>(lds, C, weight, q, n, out_action, out_logp);
                return;
            }
            // (where the fours are fewer than top_k all that is allowed is listed, and top_k
            // of them or fewer are no cut)
            if (C > (uint32_t)q.top_k) {
                by_logit = true;
                auto narrow = [&](auto each) {
                    Cut cut = find_cut(each, 0u, (uint64_t)q.top_k, [](float) { return 1u; }, lds.hist, lds.told);
                    if (q.top_p < 1.0f) {
                        uint64_t above = 0;
                        each([&](float y) {
                            if (order_key(y) > cut.key) above += weight(y);
                        });
                        above = block_sum<NW>(above, lds.sums[0]);
                        const uint64_t one = weight(key_value(cut.key));
                        uint64_t need = share(above + one * cut.ties, cut31(q.top_p));
                        if (need < 1) need = 1;
                        if (need <= above) cut = find_cut(each, cut.key, need, weight, lds.hist, lds.told);
                        else cut.ties = ties_for(need - above, one);
                    }
                    over = key_value(cut.key);
                    ties = cut.ties;
                };
                if (C <= Lds::kList)
                    narrow([&](auto f) {
                        for (uint32_t i = threadIdx.x; i < C; i += NT) f(lds.list[i]);
                    });
                else
                    narrow([&](auto f) {
                        for (int i = threadIdx.x; i < A; i += NT) f(row(i));
                    });
                over = same_in_wave(over);
                ties = same_in_wave(ties);
            }
            __syncthreads();   // top_p alone lists again
        }
    }
    // The registers come to hold the weights that are left, kTie for one equal to the cut.
    // (One pass for every kind of cut: alternatives over the registers double them.)
    const uint32_t at_cut = kFilter && by_logit ? kTie : 0u;
    uint32_t one = kFilter && by_logit ? weight(over) : 0u;   // weight of a tie
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (j < per) {
            renew(r[j]);
            if (!kFilter || vmax(j) >= over) {   // few of them hold a logit that top_k keeps
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float y = x(j, v);
                    r[j][v] = weight(y);
                    if (kFilter) r[j][v] = y > over ? r[j][v] : y == over ? at_cut : 0u;
                }
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) r[j][v] = 0u;
            }
        }
    if constexpr (kFilter) {
        if (!by_logit && q.top_p < 1.0f) {
            uint64_t sum = 0;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
#pragma unroll
                    for (int v = 0; v < V; ++v) sum += r[j][v];
                }
            for (int i = threadIdx.x; i < Lds::kBins + Lds::kBins / 16; i += NT) lds.hist[i] = 0;
            if (threadIdx.x == 0) lds.listed = 0;
            sum = block_sum<NW>(sum, lds.sums[0]);
            if (NW == 1) __syncthreads();
            uint64_t need = share(sum, cut31(q.top_p));
            if (need < 1) need = 1;
            // All weights up to `small` together stay below sum - need, so the prefix
            // ends above it.
            const uint32_t small = (uint32_t)((float)(sum - need) / (float)A * 0.999f);
            const uint32_t range = kOneBits - float_bits(small + 1);
            constexpr int kLog = NW == 1 ? 8 : 10;
            const int drop = max(0, 32 - __clz((int)range) - kLog);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (r[j][v] > small)
                            atomicAdd(&lds.hist[padded((int)((kOneBits - float_bits(r[j][v])) >> drop))],
                                      (unsigned long long)r[j][v]);
                }
            __syncthreads();
            if (wave == 0) find_bin(lds.hist, Lds::kBins, need, lds.told);
            __syncthreads();
            const uint32_t edge = same_in_wave((uint32_t)lds.told[0]);
            const uint64_t rest = same_in_wave(lds.told[1]);
            // the bin's logits (the order of logits and of weights is one, up to equal
            // weights of different logits)
            const uint32_t most = kOneBits - (edge << drop), least = most - ((1u << drop) - 1u);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const uint32_t f = float_bits(r[j][v]);
                        if (r[j][v] > small && f <= most && f >= least) {
                            const uint32_t at = atomicAdd(&lds.listed, 1u);
                            if (at < Lds::kList) lds.list[at] = row(vr.first(j) + v);
                        }
                    }
                }
            __syncthreads();
            const uint32_t C = same_in_wave(lds.listed);
            if (C <= kRank) {
                if (threadIdx.x < 4) {
                    lds.list[C + threadIdx.x] = -INFINITY;
                    lds.weight[C + threadIdx.x] = 0;
                }
                for (uint32_t i = threadIdx.x; i < C; i += NT) lds.weight[i] = weight(lds.list[i]);
                __syncthreads();
                for (uint32_t i = threadIdx.x; i < C; i += NT) {
                    const float xi = lds.list[i];
                    uint32_t equal = 0;
                    uint64_t before = 0;
                    for (uint32_t k = 0; k < C; k += 4) {
                        const float4 y = *reinterpret_cast<const float4*>(lds.list + k);
                        const uint4 w = *reinterpret_cast<const uint4*>(lds.weight + k);
                        equal += (y.x == xi) + (y.y == xi) + (y.z == xi) + (y.w == xi);
                        before += (uint64_t)(y.x > xi ? w.x : 0u) + (y.y > xi ? w.y : 0u);
                        before += (uint64_t)(y.z > xi ? w.z : 0u) + (y.w > xi ? w.w : 0u);
                    }
                    if (before < rest && rest <= before + (uint64_t)equal * lds.weight[i]) {
                        lds.told[2] = (uint64_t)__float_as_uint(xi);
                        lds.told[3] = ties_for(rest - before, lds.weight[i]);
                    }
                }
                __syncthreads();
                over = __uint_as_float(same_in_wave((uint32_t)lds.told[2]));
                ties = same_in_wave((uint32_t)lds.told[3]);
            } else {
                Cut cut;
                if (C <= Lds::kList)
                    cut = find_cut(
                        [&](auto f) {
                            for (uint32_t i = threadIdx.x; i < C; i += NT) f(lds.list[i]);
                        },
                        0u, rest, weight, lds.hist, lds.told);
                else
                    cut = find_cut(
                        [&](auto f) {
                            for (int i = threadIdx.x; i < A; i += NT) f(row(i));
                        },
                        0u, need, weight, lds.hist, lds.told);
                over = key_value(cut.key);
                ties = cut.ties;
            }
            one = weight(over);
            // another logit of the same weight: then the logits tell which are kept
            bool alike = false;
            if (C <= Lds::kList)
                for (uint32_t i = threadIdx.x; i < C; i += NT) alike |= lds.list[i] != over && weight(lds.list[i]) == one;
            else
                for (int i = threadIdx.x; i < A; i += NT) alike |= row(i) != over && weight(row(i)) == one;
            const bool ask = block_max<NW>(alike ? 1.0f : 0.0f, lds.maxima[2]) != 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        uint32_t w = r[j][v] < one ? 0u : r[j][v];
                        if (w == one) {
                            const float y = ask ? row(vr.first(j) + v) : over;
                            w = y == over ? kTie : y < over ? 0u : w;
                        }
                        r[j][v] = w;
                    }
                }
        }
    }
    if (q.least > 0) {
        if (one < q.least) one = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j < per) {
                renew(r[j]);
#pragma unroll
                for (int v = 0; v < V; ++v) r[j][v] = r[j][v] < q.least ? 0u : r[j][v];
            }
    }
    uint64_t sum = 0;
    uint32_t same = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (j < per) {
            renew(r[j]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const bool tie = kTie == r[j][v];
                same += tie;
                sum += tie ? 0u : r[j][v];
            }
        }
    sum = wave_sum(sum);
    same = wave_sum(same);
    uint64_t total, base = 0, mine;
    uint32_t left;
    if constexpr (NW == 1) {
        left = min(ties, same);
        total = mine = sum + (uint64_t)left * one;
    } else {
        if (lane == 0) {
            lds.sums[1][wave] = sum;
            lds.ties[wave] = same;
        }
        __syncthreads();
        // lane w: wave w; the ties belong to the first waves that have them
        const uint32_t has = lds.ties[lane & (NW - 1)];
        const uint32_t before = lane_scan<NW>(has, 0u, Add{}) - has;
        const uint32_t take = before < ties ? min(ties - before, has) : 0u;
        const uint64_t part = lds.sums[1][lane & (NW - 1)] + (uint64_t)take * one;
        const uint64_t run = lane_scan<NW>(part, (uint64_t)0, Add{});
        total = from_lane(run, NW - 1);
        mine = from_lane(part, wave);
        base = from_lane(run, wave) - mine;
        left = from_lane(take, wave);
    }
    const uint64_t target = share(total, cut31(q.u));
    if (base <= target && target - base < mine) {   // one wave: it walks through its part
        bool found = false;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j < per && !found) {
                renew(r[j]);
                uint32_t held = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) held += r[j][v] == kTie;
                uint32_t before = 0, inside = 0;
                if (__any(held != 0)) {
                    const uint32_t run = wave_scan(held);
                    before = run - held;
                    inside = from_lane(run, 63);
                }
                uint64_t here = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (r[j][v] == kTie) r[j][v] = before++ < left ? one : 0u;
                    here += r[j][v];
                }
                const uint64_t run = wave_scan(here);
                const uint64_t hit = __ballot(base + run > target);
                if (hit) {
                    if (lane == __ffsll((unsigned long long)hit) - 1) {
                        uint64_t c = base + run - here;
                        bool out = false;
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            c += r[j][v];
                            if (!out && c > target) {
                                out = true;
                                out_action[n] = vr.first(j) + v;
                                out_logp[n] = q.greedy ? 0.0f : logf((float)r[j][v] / (float)total);
                            }
                        }
                    }
                    found = true;
                }
                base += from_lane(run, 63);
                left -= min(left, inside);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// few actions: a row in a group of G lanes
// ---------------------------------------------------------------------------

template <int G>
__device__ __forceinline__ float group_max(float x)
{
#pragma unroll
    for (int d = G / 2; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

template <int G, class V>
__device__ __forceinline__ V group_sum(V x)
{
#pragma unroll
    for (int d = G / 2; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// Heads of up to 64 actions.  Each lane holds one action; where a filter is on, it
// counts the actions and adds the weights that come before its own, A steps.  65,536
// rows of 12: 8.2 us of kernel; 16,384 waves of 234 vector instructions, whose issue
// takes 6 us of it (some 3,700 instructions for each SIMD, four cycles each).  The
// call takes 10 to 12 us, launch and binding included; 65,536 rows of 48 with top_p 88 us,
// 48 steps each.
template <class T, int G, bool kFilter>
__global__ __launch_bounds__(kThreads) void sample_small_kernel(const Rows R, const Sampling S,
                                                                const float* __restrict__ uniform,
                                                                int64_t* __restrict__ out_action,
                                                                float* __restrict__ out_logp)
{
    const int A = R.actions, j = threadIdx.x & (G - 1), lane = threadIdx.x & 63, first = lane & ~(G - 1);
    const uint64_t group = (G == 64 ? ~0ull : (1ull << (G & 63)) - 1ull) << first;
    const int64_t step = (int64_t)gridDim.x * (kThreads / G);
    for (int64_t n0 = (int64_t)blockIdx.x * (kThreads / G); n0 < R.rows; n0 += step) {
        const int64_t n = n0 + threadIdx.x / G;
        const bool live = n < R.rows;
        const int64_t m = live ? n : R.rows - 1;
        const Row<T> row(R, m);
        const float x = j < A ? row(j) : -INFINITY;
        const float temp = S.temperatures ? S.temperatures[m] : S.temperature;
        const float u = uniform[m];
        const float top = group_max<G>(x);
        const bool bad = (__ballot(!(x < INFINITY)) & group) != 0 || !(temp >= 0.0f) || top == -INFINITY;
        const bool greedy = temp == 0.0f;   // see RowSampling
        uint32_t w = Weights(top, greedy ? 0x1p-126f : temp)(x);
        if constexpr (kFilter) {
            const int32_t k = S.top_ks ? S.top_ks[m] : S.top_k;
            const float top_p = S.top_ps ? S.top_ps[m] : S.top_p, min_p = S.min_ps ? S.min_ps[m] : S.min_p;
            int rank = 0;
            uint64_t before = 0;
            for (int i = 0; i < A; ++i) {
                const float xi = __shfl(x, first + i);
                const uint32_t wi = (uint32_t)__shfl((int)w, first + i);
                const bool ahead = xi > x || (xi == x && i < j);
                rank += ahead;
                before += ahead ? wi : 0u;
            }
            if (!greedy) {
                if (k > 0 && rank >= k) w = 0;
                if (top_p < 1.0f) {
                    const uint64_t need = share(group_sum<G>((uint64_t)w), cut31(top_p));
                    if (before >= (need < 1 ? 1 : need)) w = 0;
                }
                if (w < (uint32_t)ceilf(fminf(fmaxf(min_p, 0.0f), 1.0f) * kOne)) w = 0;
            }
        }
        if (greedy && w < 1u << 31) w = 0;
        uint64_t run = w;
#pragma unroll
        for (int d = 1; d < G; d <<= 1) {
            const uint64_t o = __shfl_up(run, d);
            if (j >= d) run += o;
        }
        const uint64_t total = __shfl(run, first + G - 1);
        const uint64_t hit = __ballot(run > share(total, greedy ? 0u : cut31(u))) & group;
        if (live && !bad && lane == __ffsll((unsigned long long)hit) - 1) {
            out_action[n] = j;
            out_logp[n] = greedy ? 0.0f : logf((float)w / (float)total);
        }
        if (live && bad && j == 0) {
            out_action[n] = -1;
            out_logp[n] = NAN;
        }
    }
}

// ---------------------------------------------------------------------------
// policy loss
// ---------------------------------------------------------------------------

// Over the workgroup; the array may be in use before.
template <int NW = kWaves, class V>
__device__ __forceinline__ V loss_sum(V x, V* lds)
{
    __syncthreads();
    return block_sum<NW>(x, lds);
}

template <int NW>
__device__ __forceinline__ float loss_max(float x, float* lds)
{
    __syncthreads();
    return block_max<NW>(x, lds);
}

// Weight of row n, 0 where it does not count.
__device__ __forceinline__ float row_weight(const Batch& b, int64_t n, int32_t A)
{
    const int64_t a = b.actions[n];
    if (a < 0 || a >= A) return 0.0f;
    return b.weights ? b.weights[n] : 1.0f;
}

// Sums of the weights, and of the advantages and their squares by weight; clears the
// count of finished workgroups that the loss kernel keeps.
static __global__ __launch_bounds__(kThreads) void loss_moments_kernel(const Batch b, int64_t rows, int32_t A,
                                                                double* __restrict__ part, uint32_t* __restrict__ done)
{
    __shared__ double lds[kWaves];
    double w0 = 0.0, w1 = 0.0, w2 = 0.0;
    for (int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x; n < rows; n += (int64_t)gridDim.x * kThreads) {
        const double w = (double)row_weight(b, n, A);
        if (w == 0.0) continue;
        const double a = (double)b.advantages[n];
        w0 += w;
        w1 += w * a;
        w2 += w * a * a;
    }
    w0 = loss_sum(w0, lds);
    w1 = loss_sum(w1, lds);
    w2 = loss_sum(w2, lds);
    if (threadIdx.x == 0) {
        part[blockIdx.x] = w0;
        part[kMomentBlocks + blockIdx.x] = w1;
        part[2 * kMomentBlocks + blockIdx.x] = w2;
        if (blockIdx.x == 0) *done = 0;
    }
}

// What all rows share: 1 / denominator, mean of the advantages, 1 / deviation.
struct Shared3 {
    float inv, mean, rstd;
};

__device__ __forceinline__ Shared3 loss_shared(const Batch& b, const double* __restrict__ part, int parts)
{
    const int lane = threadIdx.x & 63;
    double s[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] = lane < parts ? part[k * kMomentBlocks + lane] : 0.0;
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] = wave_sum(s[k]);
    Shared3 o;
    // (weights of both signs may add up to 0: no mean, but parts of a minibatch still count)
    const double den = b.denominator != 0.0f ? (double)b.denominator : s[0];
    o.inv = den != 0.0 ? (float)(1.0 / den) : 0.0f;
    o.mean = 0.0f;
    o.rstd = 1.0f;
    if (b.normalize && s[0] != 0.0) {
        const double mean = s[1] / s[0], var = s[2] / s[0] - mean * mean;
        o.mean = (float)mean;
        o.rstd = (float)(1.0 / (sqrt(var > 0.0 ? var : 0.0) + 1e-8));
    }
    return o;
}

// What a row holds apart from its logits; w is 0 where it does not count.
struct RowIn {
    float w, advantage, old_logp, value, ret, old_value;
    int32_t action;
};

__device__ __forceinline__ RowIn row_in(const Batch& b, int64_t n, int32_t A)
{
    const int64_t a = b.actions[n];
    const float w = b.weights ? b.weights[n] : 1.0f;
    const bool inside = a >= 0 && a < A;
    return RowIn{inside ? w : 0.0f, b.advantages[n], b.old_logp[n], b.values[n * b.values_stride], b.returns[n],
                 b.value_clip > 0.0f ? b.old_values[n] : 0.0f, inside ? (int32_t)a : 0};
}

// The terms of one row, given its log-probability and entropy: d loss / d log p[action]
// and d loss / d v before weights, and what goes into the sums.
struct RowTerms {
    float g, dv, sums[kSums];
};

__device__ __forceinline__ RowTerms row_terms(const Batch& b, const Shared3& s, const RowIn& in, float logp, float entropy)
{
    RowTerms o;
    const float adv = (in.advantage - s.mean) * s.rstd;
    const float diff = logp - in.old_logp;
    const float r = expf(diff);
    const float lo = 1.0f - b.clip, hi = 1.0f + b.clip;
    const float un = r * adv, cl = fminf(fmaxf(r, lo), hi) * adv;
    // (written so that a NaN stays one)
    o.sums[0] = un <= cl ? -un : cl < un ? -cl : un + cl;
    o.g = un <= cl ? -un : cl < un ? 0.0f : un + cl;
    const float v = in.value, R = in.ret;
    float err = v - R, dv = err;
    if (b.value_clip > 0.0f) {
        const float old = in.old_value, move = v - old;
        const float far = old + fminf(fmaxf(move, -b.value_clip), b.value_clip) - R;
        if (fabsf(move) > b.value_clip && fabsf(far) > fabsf(err)) {
            err = far;
            dv = 0.0f;
        }
    }
    o.dv = b.value_coef * dv;
    o.sums[1] = 0.5f * err * err;
    o.sums[2] = entropy;
    o.sums[3] = expm1f(diff) - diff;
    o.sums[4] = r < lo || r > hi ? 1.0f : 0.0f;
    return o;
}

template <int NW>
__device__ __forceinline__ void loss_stats(const Batch& b, const Shared3& s, const double* sums, int64_t blocks,
                                           double (*lds)[NW])
{
    double x[kSums] = {};
    for (int64_t i = threadIdx.x; i < blocks; i += NW * 64)
#pragma unroll
        for (int k = 0; k < kSums; ++k) x[k] += sums[i * kSums + k];
#pragma unroll
    for (int k = 0; k < kSums; ++k) x[k] = block_sum<NW>(x[k], lds[k]) * (double)s.inv;
    if (threadIdx.x == 0) {
        b.stats[0] = (float)(x[0] + (double)b.value_coef * x[1] - (double)b.entropy_coef * x[2]);
        for (int k = 0; k < kSums; ++k) b.stats[k + 1] = (float)x[k];
    }
}

// Leave this workgroup's sums; the last workgroup to do so adds them all up, in the
// order of the workgroups, and writes the statistics.  (Where a launch writes much,
// the fence that this takes in every workgroup costs more than another launch: 2,047
// rows of 16,381 in bf16 took 78 us with it and 58 with loss_stats_kernel when that was
// chosen; they take 51 to 53 now.)
template <int NW>
__device__ void loss_finish(const Batch& b, const Shared3& s, const double* acc, double* __restrict__ sums,
                            uint32_t* __restrict__ done)
{
    __shared__ uint32_t last;
    __shared__ double lds[2][kSums][NW];
    double total[kSums];
#pragma unroll
    for (int k = 0; k < kSums; ++k) total[k] = block_sum<NW>(acc[k], lds[0][k]);
    if (threadIdx.x == 0) {
        for (int k = 0; k < kSums; ++k) sums[(int64_t)blockIdx.x * kSums + k] = total[k];
        __threadfence();
        last = atomicAdd(done, 1u);
    }
    __syncthreads();
    if (last != gridDim.x - 1) return;
    __threadfence();
    loss_stats<NW>(b, s, sums, gridDim.x, lds[1]);
}

// exp d for d <= 0.  d log2 e rounded once is off by up to 2^-24 of itself, which
// the exponential of a large |d| shows; fp32 gradients take the rest of the product
// along: that of d with a constant of two terms, the first product's rounding by an fma
// (Dekker, "A floating-point technique for extending the available precision", 1971).
constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596299e-8f;   // log2 e is their sum

__device__ __forceinline__ float exp_of(float d)
{
    const float h = d * kLog2e;
    const float e = __builtin_amdgcn_exp2f(h);
    const float l = fmaf(d, kLog2eRest, fmaf(d, kLog2e, -h));
    return fmaf(e, l * 0.693147182f, e);
}

// Heads of up to 16 actions: a row to a thread.  What a row takes apart from its
// logits (the terms, two exponentials, a logarithm) is then done once for it, not by
// every lane of a group: the calls for 65,536 rows of 12 take 20 us, and
// took 42 in groups of 16 lanes (2,048 rows: 19 and 22).  17 us of it is this kernel,
// one wave to a SIMD and bound by its latencies.
template <class T>
__global__ __launch_bounds__(kThreads) void loss_thread_kernel(const Rows R, const Batch b, const Work k)
{
    constexpr int kMax = 16;
    const Shared3 s = loss_shared(b, k.part, k.parts);
    const int A = R.actions;
    const float ce = b.entropy_coef, rt = 1.0f / b.temperature;
    double acc[kSums] = {};
    for (int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x; n < R.rows; n += (int64_t)gridDim.x * kThreads) {
        const Row<T> row(R, n);
        T* out = (T*)b.dlogits + n * b.dstride;
        const RowIn in = row_in(b, n, A);
        const float w = in.w;
        if (w == 0.0f) {
            for (int i = 0; i < A; ++i) out[i] = (T)0.0f;
            b.dvalues[n] = 0.0f;
            continue;
        }
        const int a = in.action;
        float x[kMax], top = -INFINITY, xa = -INFINITY;
#pragma unroll
        for (int i = 0; i < kMax; ++i) x[i] = i < A ? row(i) : -INFINITY;
#pragma unroll
        for (int i = 0; i < kMax; ++i) {
            top = fmaxf(top, x[i]);
            xa = i == a ? x[i] : xa;
        }
        if (top == -INFINITY) top = 0.0f;   // nothing is allowed
        float e0 = 0.0f, e1 = 0.0f;
#pragma unroll
        for (int i = 0; i < kMax; ++i) {
            const float d = (x[i] - top) * rt;
            x[i] = d < -1e4f ? -1e4f : d;   // (an exponential of zero; a NaN stays one)
            const float e = exp_of(x[i]);
            e0 += e;
            e1 = fmaf(e, x[i], e1);
        }
        const float logs = logf(e0), rs = 1.0f / e0;
        const float H = e0 > 0.0f ? logs - e1 * rs : e0 == 0.0f ? 0.0f : e0;
        const RowTerms t = row_terms(b, s, in, e0 == 0.0f ? -INFINITY : (xa - top) * rt - logs, H);
        const float scale = w * s.inv;
        const float k1 = e0 == 0.0f ? 0.0f : ce * rs * scale * rt;
        const float k0 = e0 == 0.0f ? 0.0f : (ce * (H - logs) - t.g) * rs * scale * rt;
        const float ga = t.g * scale * rt;
#pragma unroll
        for (int i = 0; i < kMax; ++i)
            if (i < A) out[i] = (T)(exp_of(x[i]) * fmaf(x[i], k1, k0) + (i == a ? ga : 0.0f));
        b.dvalues[n] = t.dv * scale;
#pragma unroll
        for (int q = 0; q < kSums; ++q) acc[q] += (double)w * (double)t.sums[q];
    }
    loss_finish<kWaves>(b, s, acc, k.sums, k.done);
}

// Heads of 17 to 64 actions: a row in a group of G lanes, one action each.  65,536 rows of
// 17 take 46 us with their first launch, of 48 62 us: a row's logarithm, its two
// exponentials of ratios and the terms are computed by all lanes of the group.
template <class T, int G>
__global__ __launch_bounds__(kThreads) void loss_small_kernel(const Rows R, const Batch b, const Work k)
{
    const Shared3 s = loss_shared(b, k.part, k.parts);
    const int A = R.actions, j = threadIdx.x & (G - 1), first = threadIdx.x & 63 & ~(G - 1);
    const int64_t step = (int64_t)gridDim.x * (kThreads / G);
    const float ce = b.entropy_coef, rt = b.temperature;
    double acc[kSums] = {};
    for (int64_t n0 = (int64_t)blockIdx.x * (kThreads / G); n0 < R.rows; n0 += step) {
        const int64_t n = n0 + threadIdx.x / G;
        const bool live = n < R.rows;
        const int64_t m = live ? n : R.rows - 1;
        const RowIn in = row_in(b, m, A);
        const float w = live ? in.w : 0.0f;
        const bool on = w != 0.0f;
        const Row<T> row(R, m);
        const float x = on && j < A ? row(j) : -INFINITY;
        const int a = in.action;
        const float top = group_max<G>(x);
        const float d = x == -INFINITY ? -INFINITY : (x - top) / rt, e = expf(d);
        const float e0 = group_sum<G>(e), e1 = group_sum<G>(e != 0.0f ? e * d : 0.0f);
        const float da = __shfl(d, first + a);
        if (!live) continue;
        float y = 0.0f;
        if (on) {
            const float logs = logf(e0), rs = 1.0f / e0;
            const float H = e0 > 0.0f ? logs - e1 * rs : e0 == 0.0f ? 0.0f : e0;
            const RowTerms t = row_terms(b, s, in, e0 == 0.0f ? -INFINITY : da - logs, H);
            const float scale = w * s.inv;
            if (e != 0.0f) y = e * rs * (ce * (d - logs + H) - t.g);
            if (j == a) y += t.g;
            y = y * scale / rt;
            if (j == 0) {
                b.dvalues[n] = t.dv * scale;
#pragma unroll
                for (int q = 0; q < kSums; ++q) acc[q] += (double)w * (double)t.sums[q];
            }
        } else if (j == 0) {
            b.dvalues[n] = 0.0f;
        }
        if (j < A) ((T*)b.dlogits)[n * b.dstride + j] = (T)y;
    }
    loss_finish<kWaves>(b, s, acc, k.sums, k.done);
}

// Rows held in registers, as in sample_row_kernel: the logits are read once and the
// gradient written once.  With e = exp d and S its sum, d loss / d logit of action i is
// e_i (k1 d_i + k0), plus g at the action taken.  For 16-bit logits d is kept in units
// of log 2, so that its exponential is one instruction: rounding d there moves an
// exponential by up to 2^-24 |d| and by 2^-26 |d| for all alike (log2 e).  A 16-bit
// gradient hides that; log S and H of 16,381 normal logits are off by less than half a
// unit of fp32, as they are with a rounded (x - max) / T.  2,047 rows of 16,381 in bf16:
// 53 us with the other launches, which take 15 (64 when each load waited for the
// conversion of the one before); 4,096 of 8,191 in fp32 64 us with them (4.2 TB/s).
template <class T, int NW, int ITEMS>
__global__ __launch_bounds__(NW * 64) void loss_row_kernel(const Rows R, const Batch b, const Work k)
{
    constexpr int V = 16 / sizeof(T), NV = ITEMS / V;
    __shared__ float maxima[NW], sums[2][NW];
    __shared__ double acc[kSums];
    const Shared3 s = loss_shared(b, k.part, k.parts);
    const int A = R.actions;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr bool kHalf = sizeof(T) == 2;
    constexpr float kUnit = kHalf ? 0.693147182f : 1.0f;
    const float rt = 1.0f / b.temperature, rd = kHalf ? rt * kLog2e : rt;
    auto expd = [](float d) { return kHalf ? __builtin_amdgcn_exp2f(d) : exp_of(d); };
    if (threadIdx.x == 0)
        for (int q = 0; q < kSums; ++q) acc[q] = 0.0;
    RowIn next = (int64_t)blockIdx.x < R.rows ? row_in(b, blockIdx.x, A) : RowIn{};
    for (int64_t n = blockIdx.x; n < R.rows; n += gridDim.x) {
        const RowIn in = next;   // (the next one's numbers come while this row is worked on)
        if (n + gridDim.x < R.rows) next = row_in(b, n + gridDim.x, A);
        const VecRow<T, NW, NV, V> vr(R, n, wave, lane);
        const int per = vr.per;
        const float w = same_in_wave(in.w);
        const bool on = w != 0.0f;
        const int a = (int)same_in_wave((uint32_t)in.action);
        uint32_t r[NV][V];
        float k1 = 0.0f, k0 = 0.0f, ga = 0.0f;
        if (on) {
            const float xa = vr.row(a);
            vr.load(r);
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
#pragma unroll
                    for (int v = 0; v < V; ++v) top = fmaxf(top, __uint_as_float(r[j][v]));
                }
            top = block_max<NW>(top, maxima);
            if (top == -INFINITY) top = 0.0f;   // nothing is allowed
            // (an exponential of zero is cut off there; a NaN stays one)
            auto dist = [&](float x) {
                const float d = (x - top) * rd;
                return d < -1e4f ? -1e4f : d;
            };
            float e0 = 0.0f, e1 = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < per) {
                    renew(r[j]);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float d = dist(__uint_as_float(r[j][v])), e = expd(d);
                        e0 += e;
                        e1 = fmaf(e, d, e1);
                        r[j][v] = __float_as_uint(d);
                    }
                }
            e0 = wave_sum(e0);
            e1 = wave_sum(e1);
            if constexpr (NW > 1) {
                if (lane == 0) {
                    sums[0][wave] = e0;
                    sums[1][wave] = e1;
                }
                __syncthreads();
                e0 = from_lane(lane_scan<NW>(sums[0][lane & (NW - 1)], 0.0f, Add{}), NW - 1);
                e1 = from_lane(lane_scan<NW>(sums[1][lane & (NW - 1)], 0.0f, Add{}), NW - 1);
            }
            const float logs = logf(e0), rs = 1.0f / e0;
            const float H = e0 > 0.0f ? logs - e1 * kUnit * rs : e0 == 0.0f ? 0.0f : e0;
            const RowTerms t = row_terms(b, s, in, e0 == 0.0f ? -INFINITY : (xa - top) * rt - logs, H);
            const float scale = w * s.inv;
            k1 = e0 == 0.0f ? 0.0f : b.entropy_coef * kUnit * rs * scale * rt;
            k0 = e0 == 0.0f ? 0.0f : (b.entropy_coef * (H - logs) - t.g) * rs * scale * rt;
            ga = t.g * scale * rt;
            if (threadIdx.x == 0) {
                b.dvalues[n] = t.dv * scale;
#pragma unroll
                for (int q = 0; q < kSums; ++q) acc[q] += (double)w * (double)t.sums[q];
            }
        } else if (threadIdx.x == 0) {
            b.dvalues[n] = 0.0f;
        }
        T* out = (T*)b.dlogits + n * b.dstride;
        struct alignas(16) Vec { T v[V]; };
        const bool even = ((reinterpret_cast<uintptr_t>(out) / sizeof(T) - vr.shift) & (V - 1)) == 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j < per) {
                renew(r[j]);
                const int i0 = vr.first(j);
                Vec y;
                float z[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float d = __uint_as_float(r[j][v]);
                    z[v] = on ? expd(d) * fmaf(d, k1, k0) : 0.0f;
                }
                if (on && a >= i0 && a < i0 + V) {
#pragma unroll
                    for (int v = 0; v < V; ++v) z[v] += i0 + v == a ? ga : 0.0f;
                }
#pragma unroll
                for (int v = 0; v < V; ++v) y.v[v] = (T)z[v];
                if (even && vr.whole(j)) {
                    *reinterpret_cast<Vec*>(out + i0) = y;
                } else {
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (i0 + v >= 0 && i0 + v < A) out[i0 + v] = y.v[v];
                }
            }
        if constexpr (NW > 1) __syncthreads();
    }
    if (threadIdx.x == 0)
        for (int q = 0; q < kSums; ++q) k.sums[(int64_t)blockIdx.x * kSums + q] = acc[q];
}

// One workgroup per row, the row read again for every pass.
template <class T>
__global__ __launch_bounds__(kLongWaves * 64) void loss_long_kernel(const Rows R, const Batch b, const Work k)
{
    constexpr int NT = kLongWaves * 64;
    __shared__ float ldsf[kLongWaves];
    const Shared3 s = loss_shared(b, k.part, k.parts);
    const int A = R.actions;
    double acc[kSums] = {};
    for (int64_t n = blockIdx.x; n < R.rows; n += gridDim.x) {
        const Row<T> row(R, n);
        T* out = (T*)b.dlogits + n * b.dstride;
        const RowIn in = row_in(b, n, A);
        const float w = in.w;
        if (w == 0.0f) {
            for (int i = threadIdx.x; i < A; i += NT) out[i] = (T)0.0f;
            if (threadIdx.x == 0) b.dvalues[n] = 0.0f;
            continue;
        }
        const int a = in.action;
        float top = -INFINITY;
        walk_row(row, threadIdx.x, A, NT, [&](int, float x) { top = fmaxf(top, x); });
        const float xa = row(a);
        top = loss_max<kLongWaves>(top, ldsf);
        const float rt = b.temperature;
        // d = (x - top) / T, sum of e = exp d, and of e d
        auto dist = [&](float x) { return x == -INFINITY ? -INFINITY : (x - top) / rt; };
        float e0 = 0.0f, e1 = 0.0f;
        walk_row(row, threadIdx.x, A, NT, [&](int, float x) {
            const float d = dist(x), e = expf(d);
            e0 += e;
            if (e != 0.0f) e1 += e * d;
        });
        e0 = loss_sum<kLongWaves>(e0, ldsf);
        e1 = loss_sum<kLongWaves>(e1, ldsf);
        const float logs = logf(e0), rs = 1.0f / e0;
        const float H = e0 > 0.0f ? logs - e1 * rs : e0 == 0.0f ? 0.0f : e0;
        const RowTerms t = row_terms(b, s, in, e0 == 0.0f ? -INFINITY : dist(xa) - logs, H);
        const float scale = w * s.inv;
        const float ce = b.entropy_coef;
        walk_row(row, threadIdx.x, A, NT, [&](int i, float x) {
            const float d = dist(x), e = expf(d), p = e * rs;
            float y = e != 0.0f ? p * (ce * (d - logs + H) - t.g) : 0.0f;
            if (i == a) y += t.g;
            out[i] = (T)(y * scale / rt);
        });
        if (threadIdx.x == 0) {
            b.dvalues[n] = t.dv * scale;
            for (int q = 0; q < kSums; ++q) acc[q] += (double)w * (double)t.sums[q];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0)
        for (int q = 0; q < kSums; ++q) k.sums[(int64_t)blockIdx.x * kSums + q] = acc[q];
}

// The statistics from the sums of `blocks` workgroups, in their order.
static __global__ __launch_bounds__(kThreads) void loss_stats_kernel(const Batch b, const Work k, int64_t blocks)
{
    __shared__ double lds[kSums][kWaves];
    loss_stats<kWaves>(b, loss_shared(b, k.part, k.parts), k.sums, blocks, lds);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

namespace {

unsigned blocks_for(int64_t rows) { return (unsigned)(rows < kMaxBlocks ? rows : kMaxBlocks); }

template <int N>
using Int = std::integral_constant<int, N>;

// Waves and items of a workgroup that holds a row of so many slots in its registers.
// With many rows few waves to a row: the row's reductions take fewer barriers, and
// more rows are under way on a CU.  With fewer rows than CUs the waves are there anyway.
// fp32 in a graph, us (draws, draws with top_p, loss and gradient), by waves to a row:
//     4,096 rows of 500      one 6, 12, 19       four 11, 23, 27      sixteen 35, 112, 93
//     4,096 rows of 2,000    one 14, 28, 29      four 15, 30, 31
//     4,096 rows of 8,000    four 39, 73, 59     sixteen 50, 148, 100
//     1,024 rows of 2,000    one 7, 18, 16       four 7, 12, 15
//     1,024 rows of 16,000   four 27, 62, 33     sixteen 23, 56, 47
//       255 rows of 2,000    one 7, 16, 13       four 5, 9, 10
//       255 rows of 16,000   four 12, 28, 19     sixteen 9, 16, 17
// The 256 rows from which a row gets fewer waves are too few for draws: 256 to 512 rows
// of 1,000 to 2,000 take 1.1 to 1.9 times as long with one wave as with four (256 of 2,000
// with top_p 16.5 us and 8.8), 256 of 16,000 with top_p 29 us where sixteen take 16.
struct RowShape {
    int waves, items;
};

RowShape row_shape(int slots, int64_t rows)
{
    const bool few = rows < 256;
    if (slots <= 64 * 16 && !few) return {1, 16};
    if (slots <= 64 * 32 && !few) return {1, 32};
    if (slots <= 4 * 64 * 16) return {4, 16};
    if (slots <= 4 * 64 * 32 && !few) return {4, 32};
    if (slots <= 4 * 64 * 72 && !few) return {4, 72};
    if (slots <= 16 * 64 * 16) return {16, 16};
    if (slots <= 16 * 64 * 32) return {16, 32};
    return {16, 72};
}

// go(waves, items) with both as constants.
template <class F>
void with_shape(RowShape s, F go)
{
    auto at = [&](auto w, auto i) {
        if (s.waves == decltype(w)::value && s.items == decltype(i)::value) go(w, i);
    };
    at(Int<1>{}, Int<16>{});
    at(Int<1>{}, Int<32>{});
    at(Int<4>{}, Int<16>{});
    at(Int<4>{}, Int<32>{});
    at(Int<4>{}, Int<72>{});
    at(Int<16>{}, Int<16>{});
    at(Int<16>{}, Int<32>{});
    at(Int<16>{}, Int<72>{});
}

// Slots a row takes: rows that do not start at 16-byte addresses begin inside a vector.
template <class T>
int slots_of(const Rows& R)
{
    constexpr int V = 16 / sizeof(T);
    const bool even = aligned(R.data, 16) && (R.rows == 1 || R.stride % V == 0);
    return R.actions + (even ? 0 : V - 1);
}

}  // namespace

template <class T>
void launch_sample(const Rows& R, const Sampling& S, const float* uniform, int64_t* action, float* logp, hipStream_t s)
{
    if (R.actions <= 64) {
        const bool filter = S.top_ks || S.top_ps || S.min_ps || (S.top_k > 0 && S.top_k < R.actions) || S.top_p < 1.0f || S.min_p > 0.0f;
        const int G = group_lanes(R.actions);
        const dim3 grid(blocks_for((R.rows * G + kThreads - 1) / kThreads)), block(kThreads);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, R, S, uniform, action, logp); };
        if (filter) {
            if (G == 8) go(sample_small_kernel<T, 8, true>);
            else if (G == 16) go(sample_small_kernel<T, 16, true>);
            else if (G == 32) go(sample_small_kernel<T, 32, true>);
            else go(sample_small_kernel<T, 64, true>);
        } else {
            if (G == 8) go(sample_small_kernel<T, 8, false>);
            else if (G == 16) go(sample_small_kernel<T, 16, false>);
            else if (G == 32) go(sample_small_kernel<T, 32, false>);
            else go(sample_small_kernel<T, 64, false>);
        }
        return;
    }
    const bool filter = S.top_ks || S.top_ps || (S.top_k > 0 && S.top_k < R.actions) || S.top_p < 1.0f;
    const int slots = slots_of<T>(R);
    if (slots > kMostSlots) {
        hipLaunchKernelGGL(sample_long_kernel<T>, dim3(blocks_for(R.rows)), dim3(kLongWaves * 64), 0, s, R, S, uniform, action, logp);
        return;
    }
    const unsigned gx = blocks_for(R.rows);
    const dim3 grid(gx, (unsigned)((R.rows + gx - 1) / gx));
    with_shape(row_shape(slots, R.rows), [&](auto w, auto i) {
        constexpr int W = decltype(w)::value, I = decltype(i)::value;
        if (filter) hipLaunchKernelGGL((sample_row_kernel<T, W, I, true>), grid, dim3(W * 64), 0, s, R, S, uniform, action, logp);
        else hipLaunchKernelGGL((sample_row_kernel<T, W, I, false>), grid, dim3(W * 64), 0, s, R, S, uniform, action, logp);
    });
}

template <class T>
void launch_loss(const Rows& R, const Batch& b, const Work& k, hipStream_t s)
{
    const dim3 grid((unsigned)loss_blocks(R.rows, R.actions)), block(kThreads);
    hipLaunchKernelGGL(loss_moments_kernel, dim3((unsigned)k.parts), block, 0, s, b, R.rows, R.actions, k.part, k.done);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, R, b, k); };
    // loss_thread_kernel and loss_row_kernel multiply by 1 / T, which below 2^-128 is
    // infinite, and by which a gradient may leave fp32's range before the weight of an action
    // makes it 0.  The other two divide, last: they take the temperatures that small.
    const bool divide = b.temperature < 0x1p-64f;
    if (R.actions > 64) {
        const int slots = slots_of<T>(R);
        if (slots <= kMostSlots && !divide)
            with_shape(row_shape(slots, R.rows), [&](auto w, auto i) {
                constexpr int W = decltype(w)::value, I = decltype(i)::value;
                hipLaunchKernelGGL((loss_row_kernel<T, W, I>), grid, dim3(W * 64), 0, s, R, b, k);
            });
        else
            hipLaunchKernelGGL(loss_long_kernel<T>, grid, dim3(kLongWaves * 64), 0, s, R, b, k);
        hipLaunchKernelGGL(loss_stats_kernel, dim3(1), block, 0, s, b, k, (int64_t)grid.x);
    } else if (R.actions <= 16 && !divide) go(loss_thread_kernel<T>);
    else if (group_lanes(R.actions) <= 32) go(loss_small_kernel<T, 32>);
    else go(loss_small_kernel<T, 64>);
}

template void launch_sample<PICTURA_POLICY_TYPE>(const Rows&, const Sampling&, const float*, int64_t*, float*, hipStream_t);
template void launch_loss<PICTURA_POLICY_TYPE>(const Rows&, const Batch&, const Work&, hipStream_t);

#else   // the entries

// Workgroups of the loss: each leaves one set of partial sums, so there are no more
// than fill the card a few times.
constexpr int64_t kLossBlocks = 8192;

int64_t loss_blocks(int64_t rows, int32_t actions)
{
    const int64_t per = actions <= 16 ? kThreads : actions <= 64 ? kThreads / group_lanes(actions) : 1;
    const int64_t most = actions <= 64 ? 1024 : kLossBlocks / (actions <= 64 * 32 ? 1 : 4);
    const int64_t b = (rows + per - 1) / per;
    return b < 1 ? 1 : b < most ? b : most;
}

namespace {

size_t size_of(int32_t t) { return t == PICTURA_F32 ? 4 : 2; }

bool logits_ok(const pictura_logits* l)
{
    if (!l || (l->dtype != PICTURA_F32 && l->dtype != PICTURA_BF16 && l->dtype != PICTURA_F16)) return false;
    if (l->actions < 1 || l->actions > PICTURA_MAX_ACTIONS || l->rows < 0 || l->rows > 0x7FFFFFFFll) return false;
    if (l->rows == 0) return true;
    if (l->stride < l->actions && l->rows > 1) return false;
    if (l->mask && l->mask_stride != 0 && l->mask_stride < l->actions && l->rows > 1) return false;
    return l->data && aligned(l->data, size_of(l->dtype));
}

Rows rows_of(const pictura_logits& l) { return Rows{l.data, l.stride, l.mask, l.mask_stride, l.rows, l.actions}; }

uint64_t loss_bytes(int64_t rows, int32_t actions)
{
    return sizeof(double) * (uint64_t)(kMomentBlocks * 3 + loss_blocks(rows, actions) * kSums) + 256;
}

pictura_status launched() { return hipGetLastError() == hipSuccess ? PICTURA_OK : PICTURA_EDEVICE; }

}  // namespace
#endif
}  // namespace pictura

#ifndef PICTURA_POLICY_TYPE
using namespace pictura;

extern "C" {

pictura_status pictura_sample_actions(const pictura_logits* logits, const pictura_sampling* how, const float* uniform,
                                      int64_t* out_action, float* out_logp, void* stream)
{
    if (!logits_ok(logits) || !how) return PICTURA_EINVAL;
    if (logits->rows == 0) return PICTURA_OK;
    if (!uniform || !out_action || !out_logp || !aligned(uniform, 4) || !aligned(out_action, 8) || !aligned(out_logp, 4))
        return PICTURA_EINVAL;
    if (!aligned(how->temperatures, 4) || !aligned(how->top_ks, 4) || !aligned(how->top_ps, 4) || !aligned(how->min_ps, 4))
        return PICTURA_EINVAL;
    if (!how->temperatures && !(how->temperature >= 0.0f)) return PICTURA_EINVAL;
    if ((!how->top_ps && std::isnan(how->top_p)) || (!how->min_ps && std::isnan(how->min_p))) return PICTURA_EINVAL;
    const Sampling S{how->temperature, how->top_p, how->min_p, how->top_k,
                     how->temperatures, how->top_ps, how->min_ps, how->top_ks};
    const Rows R = rows_of(*logits);
    hipStream_t s = (hipStream_t)stream;
    if (logits->dtype == PICTURA_F32) launch_sample<float>(R, S, uniform, out_action, out_logp, s);
    else if (logits->dtype == PICTURA_BF16) launch_sample<__bf16>(R, S, uniform, out_action, out_logp, s);
    else launch_sample<_Float16>(R, S, uniform, out_action, out_logp, s);
    return launched();
}

pictura_status pictura_policy_loss_workspace(int64_t rows, int32_t actions, uint64_t* bytes)
{
    if (!bytes || rows < 0 || rows > 0x7FFFFFFFll || actions < 1 || actions > PICTURA_MAX_ACTIONS) return PICTURA_EINVAL;
    *bytes = loss_bytes(rows, actions);
    return PICTURA_OK;
}

pictura_status pictura_policy_loss(const pictura_logits* logits, const pictura_policy_batch* q, void* workspace,
                                   uint64_t workspace_bytes, float* out_stats, void* dlogits, int64_t dlogits_stride,
                                   float* dvalues, void* stream)
{
    if (!logits_ok(logits) || !q || !out_stats || !aligned(out_stats, 4) || !workspace || !aligned(workspace, 256))
        return PICTURA_EINVAL;
    if (workspace_bytes < loss_bytes(logits->rows, logits->actions)) return PICTURA_EINVAL;
    if (!(q->temperature > 0.0f) || !std::isfinite(q->temperature) || !(q->clip >= 0.0f) || std::isnan(q->value_clip) ||
        !std::isfinite(q->value_coef) || !std::isfinite(q->entropy_coef) || !(q->denominator >= 0.0f))
        return PICTURA_EINVAL;
    if (logits->rows > 0) {
        const size_t e = size_of(logits->dtype);
        if (!dlogits || !dvalues || !aligned(dlogits, e) || !aligned(dvalues, 4)) return PICTURA_EINVAL;
        if (dlogits_stride < logits->actions && logits->rows > 1) return PICTURA_EINVAL;
        if (!q->values || !q->actions || !q->old_logp || !q->advantages || !q->returns) return PICTURA_EINVAL;
        if (q->value_clip > 0.0f && !q->old_values) return PICTURA_EINVAL;
        if (!aligned(q->values, 4) || !aligned(q->actions, 8) || !aligned(q->old_logp, 4) || !aligned(q->advantages, 4) ||
            !aligned(q->returns, 4) || !aligned(q->old_values, 4) || !aligned(q->weights, 4))
            return PICTURA_EINVAL;
    }
    const Rows R = rows_of(*logits);
    const Batch b{q->values, q->values_stride, q->actions, q->old_logp, q->advantages, q->returns, q->old_values, q->weights,
                  q->temperature, q->clip, q->value_clip, q->value_coef, q->entropy_coef, q->denominator,
                  q->normalize ? 1 : 0, out_stats, dlogits, dlogits_stride, dvalues};
    hipStream_t s = (hipStream_t)stream;
    uint32_t* done = (uint32_t*)workspace;
    double* part = (double*)((char*)workspace + 256);
    const int64_t parts = R.rows / kMomentRows < 1 ? 1 : R.rows / kMomentRows < kMomentBlocks ? R.rows / kMomentRows : kMomentBlocks;
    const Work k{part, (int32_t)parts, part + 3 * kMomentBlocks, done};
    if (logits->dtype == PICTURA_F32) launch_loss<float>(R, b, k, s);
    else if (logits->dtype == PICTURA_BF16) launch_loss<__bf16>(R, b, k, s);
    else launch_loss<_Float16>(R, b, k, s);
    return launched();
}

}  // extern "C"
#endif
