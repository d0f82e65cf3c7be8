// The policy's decisions: actions drawn from logits, and the clipped policy loss
// over them with its gradient.
#include <cmath>
#include <type_traits>

#include "pictura.h"
#include "pictura_internal.h"

#pragma clang fp contract(off)

namespace pictura {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kOne = 0x1p31f;           // weight of a row's largest logit
constexpr int kMaxBlocks = 1 << 20;       // workgroups of a launch, which then take rows in turn

struct Rows {
    const void* data;
    int64_t stride;
    const uint8_t* mask;
    int64_t mask_stride;
    int64_t rows;
    int32_t actions;
};

struct Sampling {
    float temperature, top_p, min_p;
    int32_t top_k;
    const float* temperatures;
    const float* top_ps;
    const float* min_ps;
    const int32_t* top_ks;
};

// One row as the kernels read it: fp32, -inf at a place that is not allowed, and
// no negative zero (the order by bits is then that of the values).
template <class T>
struct Row {
    const T* x;
    const uint8_t* mask;
    __device__ __forceinline__ Row(const Rows& r, int64_t n)
        : x((const T*)r.data + n * r.stride), mask(r.mask ? r.mask + n * r.mask_stride : nullptr) {}
    __device__ __forceinline__ float operator()(int i) const
    {
        return mask && !mask[i] ? -INFINITY : (float)x[i] + 0.0f;
    }
};

// Bits in the order of the values.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// Weight of a logit against the row's largest.
__device__ __forceinline__ uint32_t weight_of(float x, float top, float temp)
{
    if (x == -INFINITY) return 0;
    return (uint32_t)rintf(expf((x - top) / temp) * kOne);
}

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

template <class V>
__device__ __forceinline__ V wave_sum(V x)
{
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

__device__ __forceinline__ float wave_max(float x)
{
    for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// Running sum over the wave's lanes, this one included.
template <class V>
__device__ __forceinline__ V wave_scan(V x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const V o = __shfl_up(x, d);
        if (lane >= d) x += o;
    }
    return x;
}

// Sum or maximum over a workgroup of NW waves, the same in every thread;
// lds[NW] is free again after the next barrier.
template <int NW, class V>
__device__ __forceinline__ V block_sum(V x, V* lds)
{
    x = wave_sum(x);
    if constexpr (NW == 1) return x;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int w = 1; w < NW; ++w) x += lds[w];
    return x;
}

template <int NW>
__device__ __forceinline__ float block_max(float x, float* lds)
{
    x = wave_max(x);
    if constexpr (NW == 1) return x;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int w = 1; w < NW; ++w) x = fmaxf(x, lds[w]);
    return x;
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

// First bin of `bins` (a multiple of 64) up to which the sums reach need, by one
// wave; told = {bin, need less the bins before it}.  need is at most the sum of all.
__device__ __forceinline__ void find_bin(const unsigned long long* hist, int bins, uint64_t need, uint64_t* told)
{
    const int lane = threadIdx.x & 63, per = bins / 64;
    uint64_t mine = 0;
    for (int i = 0; i < per; ++i) mine += hist[padded(lane * per + i)];
    const uint64_t run = wave_scan(mine);
    const uint64_t hit = __ballot(run >= need);
    if (lane == __ffsll((unsigned long long)hit) - 1) {
        uint64_t left = need - (run - mine);
        int i = 0;
        for (; i < per - 1; ++i) {
            const uint64_t h = hist[padded(lane * per + i)];
            if (h >= left) break;
            left -= h;
        }
        told[0] = (uint64_t)(lane * per + i);
        told[1] = left;
    }
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
    const uint64_t one = add(key_value(prefix));
    __syncthreads();
    return Cut{prefix, (uint32_t)((need + one - 1) / one)};
}

// A row's settings.
struct RowSampling {
    float temp, top_p;
    int32_t top_k;
    uint32_t least;   // smallest weight that min_p keeps
    __device__ __forceinline__ RowSampling(const Sampling& S, int64_t n)
    {
        temp = S.temperatures ? S.temperatures[n] : S.temperature;
        top_k = S.top_ks ? S.top_ks[n] : S.top_k;
        top_p = S.top_ps ? S.top_ps[n] : S.top_p;
        const float min_p = S.min_ps ? S.min_ps[n] : S.min_p;
        least = temp > 0.0f ? (uint32_t)ceilf(fminf(fmaxf(min_p, 0.0f), 1.0f) * kOne) : 0u;
    }
};

// ---------------------------------------------------------------------------
// rows of any length: read again for every pass
// ---------------------------------------------------------------------------

constexpr int kLongWaves = 16;

template <class T>
__global__ __launch_bounds__(kLongWaves * 64) void sample_long_kernel(const Rows R, const Sampling S,
                                                                      const float* __restrict__ uniform,
                                                                      int64_t* __restrict__ out_action,
                                                                      float* __restrict__ out_logp)
{
    constexpr int NW = kLongWaves, NT = NW * 64;
    __shared__ unsigned long long hist[256 + 16];
    __shared__ uint64_t told[2], lds64[NW];
    __shared__ float ldsf[NW];
    __shared__ uint32_t wties[NW];
    const int A = R.actions;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t n = blockIdx.x; n < R.rows; n += gridDim.x) {
        const Row<T> row(R, n);
        const RowSampling q(S, n);
        auto each = [&](auto f) {
            for (int i = threadIdx.x; i < A; i += NT) f(row(i));
        };
        // the largest logit; a NaN or +inf, or a temperature without meaning, makes no draw
        float top = -INFINITY, bad = q.temp >= 0.0f ? 0.0f : 1.0f;
        each([&](float x) {
            top = fmaxf(top, x);
            if (!(x < INFINITY)) bad = 1.0f;
        });
        top = block_max<NW>(top, ldsf);
        bad = block_max<NW>(bad, ldsf);
        if (bad != 0.0f || top == -INFINITY) {
            if (threadIdx.x == 0) {
                out_action[n] = -1;
                out_logp[n] = NAN;
            }
            continue;
        }
        auto weight = [&](float x) { return q.temp > 0.0f ? weight_of(x, top, q.temp) : x == top ? 1u : 0u; };
        Cut cut{0u, 0u};
        if (q.temp == 0.0f) {
            cut = Cut{order_key(top), 1u};
        } else {
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
                above = block_sum<NW>(above, lds64);
                const uint64_t one = cut.ties ? weight(key_value(cut.key)) : 0;
                uint64_t need = share(above + one * cut.ties, cut31(q.top_p));
                if (need < 1) need = 1;
                if (need <= above) cut = find_cut(each, cut.key, need, weight, hist, told);
                else cut.ties = (uint32_t)((need - above + one - 1) / one);
            }
        }
        auto kept = [&](float x) {
            const uint32_t w = weight(x);
            return w < q.least ? 0u : w;
        };
        // each wave its part of the row; the ties belong to the first waves that have them
        const int per = ((A + NT - 1) / NT) * 64, i0 = min(A, wave * per), i1 = min(A, i0 + per);
        uint64_t sum = 0;
        uint32_t ties = 0;
        for (int i = i0 + lane; i < i1; i += 64) {
            const float x = row(i);
            const uint32_t key = order_key(x);
            if (x == -INFINITY) continue;
            if (key > cut.key) sum += kept(x);
            ties += key == cut.key;
        }
        sum = wave_sum(sum);
        ties = wave_sum(ties);
        const uint32_t one = cut.ties ? kept(key_value(cut.key)) : 0u;
        __syncthreads();
        if (lane == 0) {
            lds64[wave] = sum;
            wties[wave] = ties;
        }
        __syncthreads();
        // where this wave's part of the running sum begins, and how many ties are left for it
        uint64_t total = 0, base = 0, mine = 0;
        uint32_t quota = cut.ties, left = 0;
        for (int w = 0; w < NW; ++w) {
            const uint32_t take = min(quota, wties[w]);
            const uint64_t part = lds64[w] + (uint64_t)take * one;
            if (w == wave) {
                base = total;
                mine = part;
                left = take;
            }
            quota -= take;
            total += part;
        }
        const uint64_t target = share(total, cut31(uniform[n]));
        if (base <= target && target - base < mine) {   // one wave: it walks through its part
            for (int b = i0; b < i1; b += 64) {
                const int i = b + lane;
                const float x = i < i1 ? row(i) : -INFINITY;
                const uint32_t key = order_key(x);
                const bool tie = x != -INFINITY && key == cut.key;
                const uint64_t same = __ballot(tie);
                const uint32_t before = __popcll(same & ((1ull << lane) - 1ull));
                const uint32_t w = x == -INFINITY ? 0u : key > cut.key || (tie && before < left) ? kept(x) : 0u;
                const uint64_t run = wave_scan((uint64_t)w);
                const uint64_t hit = __ballot(base + run > target);
                if (hit) {
                    if (lane == __ffsll((unsigned long long)hit) - 1) {
                        out_action[n] = i;
                        out_logp[n] = logf((float)w / (float)total);
                    }
                    break;
                }
                base += __shfl(run, 63);
                left -= min(left, (uint32_t)__popcll(same));
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

// A row of V-element vectors at 16-byte addresses: vector q covers the elements
// from q V - shift on, the first and the last only in part.
template <class T>
struct VecRow {
    static constexpr int V = 16 / sizeof(T);
    Row<T> row;
    int A, shift, vectors;
    bool mask_vec;   // the mask's bytes of a vector lie at a V-byte address
    __device__ __forceinline__ VecRow(const Rows& r, int64_t n) : row(r, n), A(r.actions)
    {
        shift = (int)(reinterpret_cast<uintptr_t>(row.x) / sizeof(T)) & (V - 1);
        vectors = (A + shift + V - 1) / V;
        mask_vec = ((reinterpret_cast<uintptr_t>(row.mask) - shift) & (V - 1)) == 0;
    }
    __device__ __forceinline__ int first(int q) const { return q * V - shift; }
    __device__ __forceinline__ void load(int q, float* x) const
    {
        const int i0 = first(q);
        if (q < vectors && i0 >= 0 && i0 + V <= A) {
            struct alignas(16) Vec { T v[V]; };
            const Vec t = *reinterpret_cast<const Vec*>(row.x + i0);
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = (float)t.v[v] + 0.0f;
            if (row.mask) {
                if (mask_vec) {
                    struct alignas(V) Bytes { uint8_t v[V]; };
                    const Bytes k = *reinterpret_cast<const Bytes*>(row.mask + i0);
#pragma unroll
                    for (int v = 0; v < V; ++v) x[v] = k.v[v] ? x[v] : -INFINITY;
                } else {
#pragma unroll
                    for (int v = 0; v < V; ++v) x[v] = row.mask[i0 + v] ? x[v] : -INFINITY;
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = q < vectors && i0 + v >= 0 && i0 + v < A ? row(i0 + v) : -INFINITY;
        }
    }
};

// One workgroup of NW waves per row, ITEMS logits to a thread, read once.  Each
// wave holds a stretch of the row, 64 vectors at a time, so that running sums by
// index go wave by wave.
template <class T, int NW, int ITEMS, bool kFilter>
__global__ __launch_bounds__(NW * 64) void sample_row_kernel(const Rows R, const Sampling S,
                                                             const float* __restrict__ uniform,
                                                             int64_t* __restrict__ out_action,
                                                             float* __restrict__ out_logp)
{
    constexpr int V = VecRow<T>::V, NV = ITEMS / V;
    constexpr int kBins = NW == 1 ? 256 : 1024, kList = NW == 1 ? 1024 : 2048;
    __shared__ unsigned long long hist[kFilter ? kBins + kBins / 16 : 1];
    __shared__ uint32_t list[kFilter ? kList : NW];
    __shared__ uint32_t listed;
    __shared__ uint64_t told[2], lds64[NW];
    __shared__ float ldsf[2 * NW];
    __shared__ uint32_t wties[NW];
    const int A = R.actions;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t n = blockIdx.x; n < R.rows; n += gridDim.x) {
        const VecRow<T> vr(R, n);
        const Row<T>& row = vr.row;
        const RowSampling q(S, n);
        const float u = uniform[n];
        const int per = (vr.vectors + NW * 64 - 1) / (NW * 64);   // vectors of a thread, at most NV
        const int q0 = wave * per * 64 + lane;                    // its first one
        float x[NV][V];
        float top = -INFINITY;
        bool odd = !(q.temp >= 0.0f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j < per) {
                vr.load(q0 + j * 64, x[j]);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) x[j][v] = -INFINITY;
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j < per) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    top = fmaxf(top, x[j][v]);
                    odd |= !(x[j][v] < INFINITY);
                }
            }
        // the largest logit; a NaN or +inf, or a temperature without meaning, makes no draw
        top = block_max<NW>(top, ldsf);
        const float bad = block_max<NW>(odd ? 1.0f : 0.0f, ldsf + NW);
        if (bad != 0.0f || top == -INFINITY) {
            if (threadIdx.x == 0) {
                out_action[n] = -1;
                out_logp[n] = NAN;
            }
            continue;
        }
        auto weight = [&](float y) { return weight_of(y, top, q.temp); };
        // Above the cut: logits over `over` and the first `ties` of those equal to it.
        // by_weight: the registers hold the weights (they keep the order of the logits, up
        // to equal ones), of which those above `wover` are kept.
        float over = -INFINITY;
        uint32_t ties = 0, wover = 0;
        bool by_weight = true;
        uint32_t (&w)[NV][V] = reinterpret_cast<uint32_t (&)[NV][V]>(x);
        if (q.temp == 0.0f) {
            over = top;
            ties = 1;
            by_weight = false;
        } else {
            Cut cut{0u, 0u};
            bool cut_k = false;
            if constexpr (kFilter) {
                uint64_t some = 0;
                if (q.top_k > 0 && q.top_k < A) {
#pragma unroll
                    for (int j = 0; j < NV; ++j)
                        if (j < per) {
#pragma unroll
                            for (int v = 0; v < V; ++v) some += x[j][v] != -INFINITY;
                        }
                    cut_k = block_sum<NW>(some, lds64) > (uint64_t)q.top_k;
                }
                if (cut_k) {
                    by_weight = false;
                    // The top_k-th largest of the vectors' maxima is no more than the top_k-th
                    // largest logit: a histogram of them bounds the logits that can be kept
                    // from below, and those few are listed.
                    float low = INFINITY;
                    float vmax[NV];
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        vmax[j] = x[j][0];
#pragma unroll
                        for (int v = 1; v < V; ++v) vmax[j] = fmaxf(vmax[j], x[j][v]);
                        if (vmax[j] > -INFINITY) low = fminf(low, vmax[j]);
                    }
                    low = -block_max<NW>(-low, ldsf);
                    const float scale = (float)kBins / (top - low);   // (no range: NaN, and all in bin 0)
                    auto bin = [&](float y) { return (int)fminf(fmaxf((top - y) * scale, 0.0f), (float)(kBins - 1)); };
                    for (int i = threadIdx.x; i < kBins + kBins / 16; i += NW * 64) hist[i] = 0;
                    if (threadIdx.x == 0) listed = 0;
                    __syncthreads();
                    uint64_t vecs = 0;
#pragma unroll
                    for (int j = 0; j < NV; ++j)
                        if (vmax[j] > -INFINITY) {
                            ++vecs;
                            atomicAdd(&hist[padded(bin(vmax[j]))], 1ull);
                        }
                    vecs = block_sum<NW>(vecs, lds64);
                    int edge = kBins - 1;
                    if (vecs >= (uint64_t)q.top_k) {
                        if (NW == 1) __syncthreads();
                        if (threadIdx.x < 64) find_bin(hist, kBins, (uint64_t)q.top_k, told);
                        __syncthreads();
                        edge = (int)told[0];
                    }
#pragma unroll
                    for (int j = 0; j < NV; ++j)
                        if (vmax[j] > -INFINITY && bin(vmax[j]) <= edge) {
#pragma unroll
                            for (int v = 0; v < V; ++v)
                                if (x[j][v] > -INFINITY && bin(x[j][v]) <= edge) {
                                    const uint32_t at = atomicAdd(&listed, 1u);
                                    if (at < kList) list[at] = __float_as_uint(x[j][v]);
                                }
                        }
                    __syncthreads();
                    const uint32_t C = listed;
                    auto from_list = [&](auto f) {
                        for (uint32_t i = threadIdx.x; i < C; i += NW * 64) f(__uint_as_float(list[i]));
                    };
                    auto from_row = [&](auto f) {
                        for (int i = threadIdx.x; i < A; i += NW * 64) f(row(i));
                    };
                    auto narrow = [&](auto each) {
                        cut = find_cut(each, 0u, (uint64_t)q.top_k, [](float) { return 1u; }, hist, told);
                        if (q.top_p < 1.0f) {
                            uint64_t above = 0;
                            each([&](float y) {
                                if (order_key(y) > cut.key) above += weight(y);
                            });
                            above = block_sum<NW>(above, lds64);
                            const uint64_t one = weight(key_value(cut.key));
                            uint64_t need = share(above + one * cut.ties, cut31(q.top_p));
                            if (need < 1) need = 1;
                            if (need <= above) cut = find_cut(each, cut.key, need, weight, hist, told);
                            else cut.ties = (uint32_t)((need - above + one - 1) / one);
                        }
                    };
                    if (C <= kList) narrow(from_list);
                    else narrow(from_row);
                    over = key_value(cut.key);
                    ties = cut.ties;
                }
            }
            if (by_weight) {
                uint64_t sum = 0;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (j < per) {
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            w[j][v] = weight(x[j][v]);
                            sum += w[j][v];
                        }
                    } else {
#pragma unroll
                        for (int v = 0; v < V; ++v) w[j][v] = 0;
                    }
                }
                if constexpr (kFilter) {
                    if (q.top_p < 1.0f) {
                        sum = block_sum<NW>(sum, lds64);
                        uint64_t need = share(sum, cut31(q.top_p));
                        if (need < 1) need = 1;
                        // All weights up to `small` together stay below sum - need, so the prefix
                        // ends above it.
                        const uint32_t small = (uint32_t)((float)(sum - need) / (float)A * 0.999f);
                        const uint32_t range = kOneBits - float_bits(small + 1);
                        constexpr int kLog = NW == 1 ? 8 : 10;
                        const int drop = max(0, 32 - __clz((int)range) - kLog);
                        auto bin = [&](uint32_t y) { return (int)((kOneBits - float_bits(y)) >> drop); };
                        for (int i = threadIdx.x; i < kBins + kBins / 16; i += NW * 64) hist[i] = 0;
                        if (threadIdx.x == 0) listed = 0;
                        __syncthreads();
#pragma unroll
                        for (int j = 0; j < NV; ++j)
                            if (j < per) {
#pragma unroll
                                for (int v = 0; v < V; ++v)
                                    if (w[j][v] > small) atomicAdd(&hist[padded(bin(w[j][v]))], (unsigned long long)w[j][v]);
                            }
                        __syncthreads();
                        if (threadIdx.x < 64) find_bin(hist, kBins, need, told);
                        __syncthreads();
                        const int edge = (int)told[0];
                        const uint64_t rest = told[1];
#pragma unroll
                        for (int j = 0; j < NV; ++j)
                            if (j < per) {
#pragma unroll
                                for (int v = 0; v < V; ++v)
                                    if (w[j][v] > small && bin(w[j][v]) == edge) {
                                        const uint32_t at = atomicAdd(&listed, 1u);
                                        if (at < kList) list[at] = (uint32_t)(vr.first(q0 + j * 64) + v);
                                    }
                            }
                        __syncthreads();
                        const uint32_t C = listed;
                        if (C <= kList) {
                            for (uint32_t i = threadIdx.x; i < C; i += NW * 64) list[i] = __float_as_uint(row((int)list[i]));
                            cut = find_cut(
                                [&](auto f) {
                                    for (uint32_t i = threadIdx.x; i < C; i += NW * 64) f(__uint_as_float(list[i]));
                                },
                                0u, rest, weight, hist, told);
                        } else {
                            cut = find_cut(
                                [&](auto f) {
                                    for (int i = threadIdx.x; i < A; i += NW * 64) f(row(i));
                                },
                                0u, need, weight, hist, told);
                        }
                        over = key_value(cut.key);
                        ties = cut.ties;
                        wover = weight(over);
                    }
                }
            }
        }
        // What is kept of element (j, v): its weight, and whether it is one of the ties.
        auto look = [&](int j, int v, uint32_t& wt, bool& tie) {
            if (by_weight) {
                const uint32_t y = w[j][v];
                wt = y > wover ? y : 0u;
                tie = false;
                if (y == wover && ties) {
                    const float z = row(vr.first(q0 + j * 64) + v);
                    if (z >= over) wt = y;
                    tie = z == over;
                }
            } else {
                const float y = x[j][v];
                tie = y == over;
                wt = 0;
                if (y >= over) wt = q.temp > 0.0f ? weight(y) : 1u;
            }
            if (wt < q.least) wt = 0;
        };
        uint64_t sum = 0;
        uint32_t same = 0, one = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j < per) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    uint32_t wt;
                    bool tie;
                    look(j, v, wt, tie);
                    if (tie) {
                        ++same;
                        one = wt;
                    } else {
                        sum += wt;
                    }
                }
            }
        sum = wave_sum(sum);
        same = wave_sum(same);
        // (of equal logits the weight is one: a wave with a tie knows it)
        for (int d = 32; d; d >>= 1) one = max(one, (uint32_t)__shfl_xor((int)one, d));
        uint64_t total = sum + (uint64_t)min(ties, same) * one, base = 0, mine = total;
        uint32_t left = min(ties, same);
        if constexpr (NW > 1) {
            __syncthreads();
            if (lane == 0) {
                lds64[wave] = sum;
                wties[wave] = same;
                list[wave] = one;
            }
            __syncthreads();
            total = 0;
            uint32_t quota = ties;
            for (int k = 0; k < NW; ++k) {
                const uint32_t take = min(quota, wties[k]);
                const uint64_t part = lds64[k] + (uint64_t)take * list[k];
                if (k == wave) {
                    base = total;
                    mine = part;
                    left = take;
                }
                quota -= take;
                total += part;
            }
        }
        const uint64_t target = share(total, cut31(u));
        if (base <= target && target - base < mine) {   // one wave: it walks through its part
            bool found = false;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (j < per && !found) {
                    uint32_t wt[V], before = 0;
                    bool tie[V];
                    uint32_t held = 0;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        look(j, v, wt[v], tie[v]);
                        held += tie[v];
                    }
                    uint32_t inside = 0;
                    if (__any(held != 0)) {
                        const uint32_t run = wave_scan(held);
                        before = run - held;
                        inside = (uint32_t)__shfl((int)run, 63);
                    }
                    uint64_t here = 0;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (tie[v] && before++ >= left) wt[v] = 0;
                        here += wt[v];
                    }
                    const uint64_t run = wave_scan(here);
                    const uint64_t hit = __ballot(base + run > target);
                    if (hit) {
                        if (lane == __ffsll((unsigned long long)hit) - 1) {
                            uint64_t c = base + run - here;
                            bool out = false;
#pragma unroll
                            for (int v = 0; v < V; ++v) {
                                c += wt[v];
                                if (!out && c > target) {
                                    out = true;
                                    out_action[n] = vr.first(q0 + j * 64) + v;
                                    out_logp[n] = logf((float)wt[v] / (float)total);
                                }
                            }
                        }
                        found = true;
                    }
                    base += __shfl(run, 63);
                    left -= min(left, inside);
                }
            }
        }
        __syncthreads();
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
// counts the actions and adds the weights that come before its own, A steps.
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
        uint32_t w;
        if (temp > 0.0f) w = weight_of(x, top, temp);
        else w = lane == __ffsll((unsigned long long)(__ballot(x == top) & group)) - 1 ? 1u : 0u;
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
            if (temp > 0.0f) {
                if (k > 0 && rank >= k) w = 0;
                if (top_p < 1.0f) {
                    const uint64_t need = share(group_sum<G>((uint64_t)w), cut31(top_p));
                    if (before >= (need < 1 ? 1 : need)) w = 0;
                }
                if (w < (uint32_t)ceilf(fminf(fmaxf(min_p, 0.0f), 1.0f) * kOne)) w = 0;
            }
        }
        uint64_t run = w;
#pragma unroll
        for (int d = 1; d < G; d <<= 1) {
            const uint64_t o = __shfl_up(run, d);
            if (j >= d) run += o;
        }
        const uint64_t total = __shfl(run, first + G - 1);
        const uint64_t hit = __ballot(run > share(total, cut31(u))) & group;
        if (live && !bad && lane == __ffsll((unsigned long long)hit) - 1) {
            out_action[n] = j;
            out_logp[n] = logf((float)w / (float)total);
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

struct Batch {
    const float* values;
    int64_t values_stride;
    const int64_t* actions;
    const float* old_logp;
    const float* advantages;
    const float* returns;
    const float* old_values;
    const float* weights;
    float temperature, clip, value_clip, value_coef, entropy_coef, denominator;
    int32_t normalize;
    float* stats;
    void* dlogits;
    int64_t dstride;
    float* dvalues;
};

constexpr int kMomentBlocks = 64;       // most partial sums of the weights and advantages: a lane each
constexpr int kMomentRows = 1024;       // rows of a workgroup that sums them, at least
constexpr int kSums = 5;                // sums over the rows: policy, value, entropy, KL, clipped

// Weight of row n, 0 where it does not count.
__device__ __forceinline__ float row_weight(const Batch& b, int64_t n, int32_t A)
{
    const int64_t a = b.actions[n];
    if (a < 0 || a >= A) return 0.0f;
    return b.weights ? b.weights[n] : 1.0f;
}

// Sums of the weights, and of the advantages and their squares by weight; clears the
// count of finished workgroups that the loss kernel keeps.
__global__ __launch_bounds__(kThreads) void loss_moments_kernel(const Batch b, int64_t rows, int32_t A,
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
    w0 = block_sum<kWaves>(w0, lds);
    w1 = block_sum<kWaves>(w1, lds);
    w2 = block_sum<kWaves>(w2, lds);
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
    const double den = b.denominator != 0.0f ? (double)b.denominator : s[0];
    o.inv = s[0] != 0.0 ? (float)(1.0 / den) : 0.0f;
    o.mean = 0.0f;
    o.rstd = 1.0f;
    if (b.normalize && s[0] != 0.0) {
        const double mean = s[1] / s[0], var = s[2] / s[0] - mean * mean;
        o.mean = (float)mean;
        o.rstd = (float)(1.0 / (sqrt(var > 0.0 ? var : 0.0) + 1e-8));
    }
    return o;
}

// The terms of one row, given its log-probability and entropy: d loss / d log p[action]
// and d loss / d v before weights, and what goes into the sums.
struct RowTerms {
    float g, dv, sums[kSums];
};

__device__ __forceinline__ RowTerms row_terms(const Batch& b, const Shared3& s, int64_t n, float logp, float entropy)
{
    RowTerms o;
    const float adv = (b.advantages[n] - s.mean) * s.rstd;
    const float diff = logp - b.old_logp[n];
    const float r = expf(diff);
    const float lo = 1.0f - b.clip, hi = 1.0f + b.clip;
    const float un = r * adv, cl = fminf(fmaxf(r, lo), hi) * adv;
    // (written so that a NaN stays one)
    o.sums[0] = un <= cl ? -un : cl < un ? -cl : un + cl;
    o.g = un <= cl ? -un : cl < un ? 0.0f : un + cl;
    const float v = b.values[n * b.values_stride], R = b.returns[n];
    float err = v - R, dv = err;
    if (b.value_clip > 0.0f) {
        const float old = b.old_values[n], move = v - old;
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

// Leave this workgroup's sums; the last workgroup to do so adds them all up, in the
// order of the workgroups, and writes the statistics.
__device__ void loss_finish(const Batch& b, const Shared3& s, const double* acc, double* __restrict__ sums,
                            uint32_t* __restrict__ done, double* lds)
{
    __shared__ uint32_t last;
    double total[kSums];
#pragma unroll
    for (int k = 0; k < kSums; ++k) total[k] = block_sum<kWaves>(acc[k], lds);
    if (threadIdx.x == 0) {
        for (int k = 0; k < kSums; ++k) sums[(int64_t)blockIdx.x * kSums + k] = total[k];
        __threadfence();
        last = atomicAdd(done, 1u);
    }
    __syncthreads();
    if (last != gridDim.x - 1) return;
    __threadfence();
    double x[kSums] = {};
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads)
#pragma unroll
        for (int k = 0; k < kSums; ++k) x[k] += sums[(int64_t)i * kSums + k];
#pragma unroll
    for (int k = 0; k < kSums; ++k) x[k] = block_sum<kWaves>(x[k], lds) * (double)s.inv;
    if (threadIdx.x == 0) {
        b.stats[0] = (float)(x[0] + (double)b.value_coef * x[1] - (double)b.entropy_coef * x[2]);
        for (int k = 0; k < kSums; ++k) b.stats[k + 1] = (float)x[k];
    }
}

struct Work {
    const double* part;   // sums of loss_moments_kernel
    int32_t parts;
    double* sums;
    uint32_t* done;
};

// Heads of up to 64 actions: a row in a group of G lanes, one action each.
template <class T, int G>
__global__ __launch_bounds__(kThreads) void loss_small_kernel(const Rows R, const Batch b, const Work k)
{
    __shared__ double lds[kWaves];
    const Shared3 s = loss_shared(b, k.part, k.parts);
    const int A = R.actions, j = threadIdx.x & (G - 1), first = threadIdx.x & 63 & ~(G - 1);
    const int64_t step = (int64_t)gridDim.x * (kThreads / G);
    const float ce = b.entropy_coef, rt = b.temperature;
    double acc[kSums] = {};
    for (int64_t n0 = (int64_t)blockIdx.x * (kThreads / G); n0 < R.rows; n0 += step) {
        const int64_t n = n0 + threadIdx.x / G;
        const bool live = n < R.rows;
        const int64_t m = live ? n : R.rows - 1;
        const float w = live ? row_weight(b, m, A) : 0.0f;
        const bool on = w != 0.0f;
        const Row<T> row(R, m);
        const float x = on && j < A ? row(j) : -INFINITY;
        const int a = on ? (int)b.actions[m] : 0;
        const float top = group_max<G>(x);
        const float d = x == -INFINITY ? -INFINITY : (x - top) / rt, e = expf(d);
        const float e0 = group_sum<G>(e), e1 = group_sum<G>(e != 0.0f ? e * d : 0.0f);
        const float da = __shfl(d, first + a);
        if (!live) continue;
        float y = 0.0f;
        if (on) {
            const float logs = logf(e0), rs = 1.0f / e0;
            const float H = e0 > 0.0f ? logs - e1 * rs : e0 == 0.0f ? 0.0f : e0;
            const RowTerms t = row_terms(b, s, m, e0 == 0.0f ? -INFINITY : da - logs, H);
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
    loss_finish(b, s, acc, k.sums, k.done, lds);
}

// One workgroup per row, the row read again for every pass.
template <class T>
__global__ __launch_bounds__(kThreads) void loss_kernel(const Rows R, const Batch b, const Work k)
{
    __shared__ double ldsd[kWaves];
    __shared__ float ldsf[kWaves];
    const Shared3 s = loss_shared(b, k.part, k.parts);
    const int A = R.actions;
    double acc[kSums] = {};
    for (int64_t n = blockIdx.x; n < R.rows; n += gridDim.x) {
        const Row<T> row(R, n);
        T* out = (T*)b.dlogits + n * b.dstride;
        const float w = row_weight(b, n, A);
        if (w == 0.0f) {
            for (int i = threadIdx.x; i < A; i += kThreads) out[i] = (T)0.0f;
            if (threadIdx.x == 0) b.dvalues[n] = 0.0f;
            continue;
        }
        const int a = (int)b.actions[n];
        float top = -INFINITY;
        for (int i = threadIdx.x; i < A; i += kThreads) top = fmaxf(top, row(i));
        const float xa = row(a);
        top = block_max<kWaves>(top, ldsf);
        const float rt = b.temperature;
        // d = (x - top) / T, sum of e = exp d, and of e d
        auto dist = [&](float x) { return x == -INFINITY ? -INFINITY : (x - top) / rt; };
        float e0 = 0.0f, e1 = 0.0f;
        for (int i = threadIdx.x; i < A; i += kThreads) {
            const float d = dist(row(i)), e = expf(d);
            e0 += e;
            if (e != 0.0f) e1 += e * d;
        }
        e0 = block_sum<kWaves>(e0, ldsf);
        e1 = block_sum<kWaves>(e1, ldsf);
        const float logs = logf(e0), rs = 1.0f / e0;
        const float H = e0 > 0.0f ? logs - e1 * rs : e0 == 0.0f ? 0.0f : e0;
        const RowTerms t = row_terms(b, s, n, e0 == 0.0f ? -INFINITY : dist(xa) - logs, H);
        const float scale = w * s.inv;
        const float ce = b.entropy_coef;
        for (int i = threadIdx.x; i < A; i += kThreads) {
            const float d = dist(row(i)), e = expf(d), p = e * rs;
            float y = e != 0.0f ? p * (ce * (d - logs + H) - t.g) : 0.0f;
            if (i == a) y += t.g;
            out[i] = (T)(y * scale / rt);
        }
        if (threadIdx.x == 0) {
            b.dvalues[n] = t.dv * scale;
            for (int q = 0; q < kSums; ++q) acc[q] += (double)w * (double)t.sums[q];
        }
        __syncthreads();
    }
    loss_finish(b, s, acc, k.sums, k.done, ldsd);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

namespace {

size_t size_of(int32_t t) { return t == PICTURA_F32 ? 4 : 2; }

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

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

unsigned blocks_for(int64_t rows) { return (unsigned)(rows < kMaxBlocks ? rows : kMaxBlocks); }

// Lanes that hold a row of up to 64 actions.
int group_lanes(int32_t actions) { return actions <= 8 ? 8 : actions <= 16 ? 16 : actions <= 32 ? 32 : 64; }

// Workgroups of the loss: each leaves one set of partial sums.
constexpr int64_t kLossBlocks = 4096;

int64_t loss_blocks(int64_t rows, int32_t actions)
{
    const int64_t per = actions <= 64 ? kThreads / group_lanes(actions) : 1;
    const int64_t b = (rows + per - 1) / per;
    return b < 1 ? 1 : b < kLossBlocks ? b : kLossBlocks;
}

uint64_t loss_bytes(int64_t rows, int32_t actions)
{
    return sizeof(double) * (uint64_t)(kMomentBlocks * 3 + loss_blocks(rows, actions) * kSums) + 256;
}

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
    // slots a row takes: rows that do not start at 16-byte addresses begin inside a vector
    constexpr int V = 16 / sizeof(T);
    const bool even = aligned(R.data, 16) && (R.rows == 1 || R.stride % V == 0);
    const int slots = R.actions + (even ? 0 : V - 1);
    const dim3 grid(blocks_for(R.rows));
    auto go = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, grid, dim3(waves * 64), 0, s, R, S, uniform, action, logp);
    };
    auto pick = [&](auto f) {
        constexpr bool F = decltype(f)::value;
        if (slots <= 64 * 16) go(sample_row_kernel<T, 1, 16, F>, 1);
        else if (slots <= 4 * 64 * 16) go(sample_row_kernel<T, 4, 16, F>, 4);
        else if (slots <= 4 * 64 * 32) go(sample_row_kernel<T, 4, 32, F>, 4);
        else if (slots <= 16 * 64 * 16) go(sample_row_kernel<T, 16, 16, F>, 16);
        else if (slots <= 16 * 64 * 32) go(sample_row_kernel<T, 16, 32, F>, 16);
        else if (slots <= 16 * 64 * 72) go(sample_row_kernel<T, 16, 72, F>, 16);
        else go(sample_long_kernel<T>, kLongWaves);
    };
    if (filter) pick(std::true_type{});
    else pick(std::false_type{});
}

template <class T>
void launch_loss(const Rows& R, const Batch& b, const Work& k, hipStream_t s)
{
    const dim3 grid((unsigned)loss_blocks(R.rows, R.actions)), block(kThreads);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, R, b, k); };
    if (R.actions > 64) go(loss_kernel<T>);
    else if (group_lanes(R.actions) == 8) go(loss_small_kernel<T, 8>);
    else if (group_lanes(R.actions) == 16) go(loss_small_kernel<T, 16>);
    else if (group_lanes(R.actions) == 32) go(loss_small_kernel<T, 32>);
    else go(loss_small_kernel<T, 64>);
}

pictura_status launched() { return hipGetLastError() == hipSuccess ? PICTURA_OK : PICTURA_EDEVICE; }

}  // namespace
}  // namespace pictura

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
    hipLaunchKernelGGL(loss_moments_kernel, dim3((unsigned)parts), dim3(kThreads), 0, s, b, R.rows, R.actions, part, done);
    if (logits->dtype == PICTURA_F32) launch_loss<float>(R, b, k, s);
    else if (logits->dtype == PICTURA_BF16) launch_loss<__bf16>(R, b, k, s);
    else launch_loss<_Float16>(R, b, k, s);
    return launched();
}

}  // extern "C"
