// A memory over the steps of sequences: the gated linear recurrence
//     a = sigmoid(g),  h_t = a_t h_(t-1) + (1 - a_t) x_t
// per channel (h_(t-1) taken as 0 where a step is reset), its gradient, and one step
// of it in place.
//
// Gradient.  With G_t the gradient of h_t, all later steps included, and c_t = a_t G_t
// what step t hands back (0 at a reset):
//     G_t = dout_t + c_(t+1),  dx_t = (1 - a_t) G_t,  dg_t = a_t (1 - a_t) (h_(t-1) - x_t) G_t,
// the same recurrence backwards.  h_(t-1) is needed in fp32: the forward pass leaves the
// state before every 16th step, and the steps between are computed again in registers
// (0.25 byte an element instead of 4).
//
// A thread walks through the steps of one or two channels, 16 steps' loads under way at
// once.  Where there are too few channels for the card, the steps are cut into tiles, a
// workgroup each: what a tile's steps do to a state is h -> P h + H, with P the product of
// their a, which every workgroup tells those behind it; it keeps a and (1 - a) x in registers
// until it knows the state before its own (a scan in one pass with a look back: Merrill and
// Garland, "Single-pass parallel prefix scan with decoupled look-back", 2016; here by groups of
// tiles, and values that carry their own flag).  Everything is read and written once, and joined
// in one order, so that results repeat to the bit.
//
// Measured (one MI355X, large copies at 5,150 GB/s): 2,048 x 128 steps of 512 channels in bf16
// forward 173 to 179 us, gradient 294 (838 and 1,376 MB with the saved states: 4.7 and 4.7 TB/s,
// the gradient with four registers spilled where there are no resets); one
// of 65,521 steps of 1,024 forward 109 us, gradient 160 (419 and 688 MB: 3.8 and 4.3 TB/s), of
// which a launch that sums the segments up first and one that reads them again took 152 and 221;
// single steps of 65,536 x 512 in bf16 69 us (470 MB: 6.8 TB/s, some of it from the caches).
#include <cmath>

#include "pictura.h"
#include "pictura_internal.h"
#include "pictura_overlap.h"

#pragma clang fp contract(off)

namespace pictura {
namespace {

constexpr int kSteps = PICTURA_SCAN_STEPS;   // steps between saved states, and in registers at once

// Neighbouring channels, loaded and stored as one at any address.
template <class T, int V>
struct Vec {
    T v[V];
};

template <class T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p)
{
    Vec<T, V> x;
    __builtin_memcpy(&x, p, sizeof(x));
    return x;
}

template <class T, int V>
__device__ __forceinline__ void store(T* p, const Vec<T, V>& x) { __builtin_memcpy(p, &x, sizeof(x)); }

// Element (b, t, c) of a sequence's tensor is at data[b * batch + t * step + c].
template <class T>
struct Tensor {
    T* data;
    int64_t batch, step;
};

template <class T>
struct Sequences {
    Tensor<const T> gates, inputs;
    const float* state;                 // [batch][channels]
    Tensor<const uint8_t> resets;       // one channel
    int64_t threads, steps;             // vectors of channels in all, steps
    int64_t states;                     // channels in all
    int32_t channels, vectors;          // of a sequence, and the vectors that cover them
    bool one;                           // a wave's are of one sequence
};

// The smaller one of a = sigmoid(g) and 1 - a, with g's sign: the other one is 1 - |m| to half
// a unit.  For fp32, e = exp(-|g|) takes the product by log2(e) in two terms (at 128 and
// beyond it is 0): e is off by up to 3.5 u (u = 2^-24), the reciprocal by 4.5 u, m by 8.5 u.
// 16-bit gates take the product in one, off by 1.3 |g| u more: where |g| is large m is small,
// so that a and 1 - a stay within half a unit of 1, and their inputs are rounded to 2^-9 or
// 2^-12 of themselves.  Tiles of bf16 are bound by the vector unit: forward over one of 65,536
// steps of 1,024 channels takes 121 us with two terms.
template <class T>
__device__ __forceinline__ float gate_of(float g)
{
    constexpr float kHi = 1.44269502f, kLo = 1.92596299e-8f, kLn2 = 0.693147182f;
    float e;
    if constexpr (sizeof(T) == 2) {
        e = __builtin_amdgcn_exp2f(fabsf(g) * -kHi);
    } else {
        const float z = fabsf(g) > 128.0f ? 128.0f : fabsf(g);   // (a NaN stays one)
        const float hi = z * -kHi, lo = fmaf(z, -kLo, fmaf(z, -kHi, -hi));
        e = __builtin_amdgcn_exp2f(hi);
        e = fmaf(e * lo, kLn2, e);
    }
    return copysignf(e * __builtin_amdgcn_rcpf(1.0f + e), g);
}

// m as a and b = 1 - a.
__device__ __forceinline__ void gate_parts(float m, float& a, float& b)
{
    const float s = fabsf(m), l = 1.0f - s;
    const bool negative = __float_as_uint(m) >> 31;
    a = negative ? s : l;
    b = negative ? l : s;
}

// What steps do to a state, h -> P h + H.  A reset among them makes P -0 (every other
// product is +0 or more): the state does not count then, even if it is a NaN.
struct Map {
    float P, H;
};

__device__ __forceinline__ float apply(const Map& f, float h)
{
    return __float_as_uint(f.P) == 0x80000000u ? f.H : fmaf(f.P, h, f.H);
}

// f, then g
__device__ __forceinline__ Map then(const Map& f, const Map& g)
{
    return Map{__float_as_uint(g.P) == 0x80000000u ? g.P : g.P * f.P, apply(g, f.H)};
}

// A product of gates as others may use it: what fp32 does not reach is 2^-149, the smallest number
// above 0, and not 0.  An infinite state then stays infinite, as it does through the steps one by
// one, where 0 times infinity is a NaN; of a finite one it is off by 2^-149, as products next to it
// are.  (As whole numbers: -0 and NaN are larger.)
__device__ __forceinline__ float kept(float P) { return __uint_as_float(max(__float_as_uint(P), 1u)); }

// Says that x may be new from here on, and in this order: what is computed from it is not
// computed earlier, where it would take registers for longer.
__device__ __forceinline__ void hold(float& x) { asm volatile("" : "+v"(x)); }

template <class T, int V>
__device__ __forceinline__ void hold(Vec<T, V>& x)
{
    if constexpr (sizeof(x) == 4) {
        uint32_t w = __builtin_bit_cast(uint32_t, x);
        asm volatile("" : "+v"(w));
        x = __builtin_bit_cast(Vec<T, V>, w);
    }
}

// Where a thread's channels begin in the tensors, and among all channels.  Where a sequence's
// channels are no multiple of V the last vector begins earlier, and two threads compute
// and write the same for what both hold.
template <class T, int V>
struct Place {
    int64_t b, flat;
    int32_t c;
    __device__ __forceinline__ Place(int64_t thread, int32_t vectors, int32_t channels)
    {
        int32_t i;
        if (thread >> 32 == 0) {   // (a 64-bit division takes some hundred instructions)
            b = (uint32_t)thread / (uint32_t)vectors;
            i = (int32_t)((uint32_t)thread % (uint32_t)vectors);
        } else {
            b = thread / vectors;
            i = (int32_t)(thread % vectors);
        }
        c = min(i * V, channels - V);
        flat = b * channels + c;
    }
    template <class U>
    __device__ __forceinline__ U* in(const Tensor<U>& x) const { return x.data + b * x.batch + c; }
    __device__ __forceinline__ const uint8_t* flags(const Tensor<const uint8_t>& x) const { return x.data + b * x.batch; }
};

// Up to N steps of a tensor; those from n on are zeros.
template <class T, int V, int N>
__device__ __forceinline__ void load_steps(const T* p, int64_t step, int n, Vec<T, V> (&x)[N])
{
    if (n == N) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = load<T, V>(p + i * step);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = Vec<T, V>{};
            if (i < n) x[i] = load<T, V>(p + i * step);
        }
    }
}

// Bit i: whether step i of n is reset.  Where a wave's channels are all of one sequence,
// each of its lanes looks at one step.
template <bool kResets, int N>
__device__ __forceinline__ uint32_t load_resets(const uint8_t* p, int64_t step, int n, bool one)
{
    uint32_t bits = 0;
    if constexpr (kResets) {
        if (one) {
            const int lane = threadIdx.x & 63;
            return (uint32_t)__ballot(lane < n && p[lane * step] != 0);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n && p[i * step]) bits |= 1u << i;
    }
    return bits;
}

// Waves of a tile, kSteps steps each: two channels a thread leave registers for two
// workgroups of eight on a CU (one of 65,536 steps of 1,024 in bf16: forward 120 us, gradient
// 173; with sixteen 120 and 180, with four 158 and 237; all before gates of 16
// bits took their exponential in one product), one channel for two of sixteen
// (three of 8,192 of 330 in fp32: 30 and 43 us; with eight 37 and 45).
constexpr int tile_waves(int vec) { return vec == 2 ? 8 : 16; }
constexpr int tile_steps(int vec) { return tile_waves(vec) * kSteps; }

template <int V>
struct alignas(8 * V) Maps {
    Map v[V];
};

// ---------------------------------------------------------------------------
// few channels: the steps cut into tiles, a workgroup each
// ---------------------------------------------------------------------------

// What workgroups tell one another: a 64-bit word that holds a value together with the
// fact that it is there, so that it needs no fence.  `tiles` has P and H of every tile, with
// P in the lower half, which is kEmpty before; `groups` the state after every kGroup tiles in
// the upper half of a word whose lower half is kEmpty before.
constexpr uint32_t kEmpty = 0xFFFFFFFFu;
constexpr int kGroup = 16;                       // tiles of a group
constexpr int kPolls = 1 << 20;                  // of a wait, a second or more

typedef unsigned long long Word;

struct Chain {
    uint32_t* ticket;
    Word* tiles;    // [tiles][threads][V]
    Word* groups;   // [groups][threads][V]
    int64_t words;  // of both
    int32_t count;  // tiles
};

__device__ __forceinline__ void tell(Word* at, uint32_t low, float high)
{
    __hip_atomic_store(at, (Word)__float_as_uint(high) << 32 | low, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void tell(Word* at, const Map& m)
{
    const uint32_t p = __float_as_uint(m.P);
    tell(at, p == kEmpty ? 0x7FC00000u : p, m.H);   // (a NaN of that pattern: any other)
}

template <int V>
constexpr int kItems = kGroup / tile_waves(V);   // tiles of its group that a wave waits for

// Waits until the words of up to kItems<V> tiles are there, `apart` of them apart.  A workgroup
// waits only for such with smaller tickets, which have started before it and in turn wait
// only for smaller ones: every wait ends, long before kPolls.  (If one did not, its values would
// be taken as they are: NaN states from there to the next reset, as the header says.)
template <int V>
__device__ __forceinline__ void await(const Word* at, int64_t apart, int items, bool on, Word (&w)[kItems<V>][V])
{
    for (int i = 0; i < kPolls; ++i) {
        bool there = true;
#pragma unroll
        for (int k = 0; k < kItems<V>; ++k)
            if (k < items) {
#pragma unroll
                for (int v = 0; v < V; ++v) w[k][v] = on ? __hip_atomic_load(at + k * apart + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
            }
#pragma unroll
        for (int k = 0; k < kItems<V>; ++k)
            if (k < items) {
#pragma unroll
                for (int v = 0; v < V; ++v) there = there && (uint32_t)w[k][v] != kEmpty;
            }
        if (__all(there)) return;
        __builtin_amdgcn_s_sleep(1);
    }
}

// Clears what the workgroups of one call tell one another.
static __global__ __launch_bounds__(256) void chain_kernel(const Chain c)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i == 0) *c.ticket = 0;
    if (i < c.words) c.tiles[i] = ~0ull;
}

template <int V>
struct TileLds {
    Maps<V> waves[tile_waves(V)][64];   // of this tile
    Maps<V> before[kGroup][64];         // of the tiles before it in its group
    float start[64][V];                 // the state before the group
    uint32_t ticket;
};

// This workgroup's tile and channels, in the order in which workgroups start: all channels
// of a tile before the next one.
template <int V>
__device__ __forceinline__ int32_t take_ticket(const Chain& c, TileLds<V>& lds, int32_t blocks, int32_t& block)
{
    if (threadIdx.x == 0) lds.ticket = atomicAdd(c.ticket, 1u);
    __syncthreads();
    block = (int32_t)(lds.ticket % (uint32_t)blocks);
    return (int32_t)(lds.ticket / (uint32_t)blocks);
}

// The state before this wave's steps.  k: the tile in the order of the recurrence, w: the
// wave in that order, f: what its steps do; first: the state before tile 0.
template <int V>
__device__ __forceinline__ void state_before(const Chain& c, TileLds<V>& lds, int64_t threads, int64_t thread, bool on, int32_t k,
                                             int w, const Maps<V>& f, const float (&first)[V], float (&h)[V])
{
    constexpr int W = tile_waves(V);
    const int lane = threadIdx.x & 63;
    const int32_t g = k / kGroup, r = k % kGroup;
    lds.waves[w][lane] = f;
    __syncthreads();
    if (w == W - 1 && r < kGroup - 1 && k < c.count - 1) {   // what the whole tile does
        Maps<V> all = lds.waves[0][lane];
#pragma unroll 2
        for (int i = 1; i < W; ++i) {
            const Maps<V> m = lds.waves[i][lane];
#pragma unroll
            for (int v = 0; v < V; ++v) all.v[v] = then(all.v[v], m.v[v]);
        }
        if (on) {
#pragma unroll
            for (int v = 0; v < V; ++v) tell(c.tiles + ((int64_t)k * threads + thread) * V + v, Map{kept(all.v[v].P), all.v[v].H});
        }
    }
    // each wave waits for some of the tiles before
    Maps<V> m;
    const int mine = min(kItems<V>, r - w * kItems<V>);
    if (mine > 0) {
        Word x[kItems<V>][V];
        await<V>(c.tiles + ((int64_t)(g * kGroup + w * kItems<V>) * threads + thread) * V, threads * V, mine, on, x);
#pragma unroll
        for (int i = 0; i < kItems<V>; ++i)
            if (i < mine) {
#pragma unroll
                for (int v = 0; v < V; ++v) m.v[v] = Map{__uint_as_float((uint32_t)x[i][v]), __uint_as_float((uint32_t)(x[i][v] >> 32))};
                lds.before[w * kItems<V> + i][lane] = m;
            }
    }
    __syncthreads();
    // The last wave waits for the state before the group.  In a group's last tile it has joined
    // all of the group by then: from one group to the next there is one wait and one product.
    if (w == W - 1) {
        const bool ends = r == kGroup - 1 && k < c.count - 1;
        if (ends) {
            m = lds.before[0][lane];
#pragma unroll 4
            for (int i = 1; i < kGroup - 1 + W; ++i) {
                const Maps<V> n = i < kGroup - 1 ? lds.before[i][lane] : lds.waves[i - (kGroup - 1)][lane];
#pragma unroll
                for (int v = 0; v < V; ++v) m.v[v] = then(m.v[v], n.v[v]);
            }
        }
        float start[V];
        Word x[kItems<V>][V];
        if (g > 0) await<V>(c.groups + ((int64_t)(g - 1) * threads + thread) * V, 0, 1, on, x);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            start[v] = g > 0 ? __uint_as_float((uint32_t)(x[0][v] >> 32)) : first[v];
            if (ends && on) tell(c.groups + ((int64_t)g * threads + thread) * V + v, 0u, apply(Map{kept(m.v[v].P), m.v[v].H}, start[v]));
            lds.start[lane][v] = start[v];
        }
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = lds.start[lane][v];
#pragma unroll 4
    for (int i = 0; i < r; ++i) {
        m = lds.before[i][lane];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = apply(m.v[v], h[v]);
    }
#pragma unroll 4
    for (int i = 0; i < w; ++i) {
        m = lds.waves[i][lane];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = apply(m.v[v], h[v]);
    }
}

// Forwards over one tile.  Of bf16 it takes 940 vector instructions a wave, and the vector units
// are busy for 55 % of its time (backwards 1,520 and 60 %); workgroups that take several tiles, and the next ticket ahead, are slower (169 us and
// 121), as tickets wait for workgroups that are not ready.
template <class T, int V, bool kResets>
__global__ __launch_bounds__(tile_waves(V) * 64, 4) void tile_kernel(const Sequences<T> q, const Tensor<T> out, float* __restrict__ last,
                                                                  float* __restrict__ saved, const Chain chain)
{
    __shared__ TileLds<V> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t block;
    const int32_t tile = take_ticket<V>(chain, lds, (int32_t)((q.threads + 63) / 64), block);
    const int64_t thread = (int64_t)block * 64 + lane;
    const bool on = thread < q.threads;
    const Place<T, V> at(on ? thread : 0, q.vectors, q.channels);   // (lanes beyond the last channel read the first ones' and write nothing)
    const int64_t t = (int64_t)tile * tile_steps(V) + wave * kSteps;
    const int n = (int)max((int64_t)0, min((int64_t)kSteps, q.steps - t));
    float a[kSteps][V], add[kSteps][V], first[V], h[V];
    uint32_t resets;
    Maps<V> f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        f.v[v] = Map{1.0f, 0.0f};
        first[v] = q.state && on ? q.state[at.flat + v] : 0.0f;
    }
    {
        Vec<T, V> gs[kSteps], xs[kSteps];
        load_steps<T, V>(at.in(q.gates) + t * q.gates.step, q.gates.step, n, gs);
        load_steps<T, V>(at.in(q.inputs) + t * q.inputs.step, q.inputs.step, n, xs);
        resets = load_resets<kResets, kSteps>(at.flags(q.resets) + t * q.resets.step, q.resets.step, n, q.one);
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float b;
                gate_parts(gate_of<T>((float)gs[i].v[v]), a[i][v], b);
                add[i][v] = b * (float)xs[i].v[v];
                const bool reset = kResets && (resets >> i & 1u);
                Map& m = f.v[v];
                if (i < n) {
                    m.H = reset ? add[i][v] : fmaf(a[i][v], m.H, add[i][v]);
                    m.P = reset ? -0.0f : a[i][v] * m.P;   // (-0 stays -0)
                }
                hold(a[i][v]);
                hold(add[i][v]);
            }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) f.v[v].P = kept(f.v[v].P);
    state_before<V>(chain, lds, q.threads, thread, on, tile, wave, f, first, h);
    if (!on || n == 0) return;
    if (saved) {
        Vec<float, V> s;
#pragma unroll
        for (int v = 0; v < V; ++v) s.v[v] = h[v];
        store<float, V>(saved + (t / kSteps) * q.states + at.flat, s);
    }
    T* y = at.in(out) + t * out.step;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (i >= n) continue;
        Vec<T, V> o;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            h[v] = kResets && (resets >> i & 1u) ? add[i][v] : fmaf(a[i][v], h[v], add[i][v]);
            o.v[v] = (T)h[v];
        }
        store<T, V>(y + i * out.step, o);
    }
    if (last && t + n == q.steps) {
#pragma unroll
        for (int v = 0; v < V; ++v) last[at.flat + v] = h[v];
    }
}

// Backwards over one tile, from the last one on.
template <class T, int V, bool kResets>
__global__ __launch_bounds__(tile_waves(V) * 64, 4) void tile_gradient_kernel(const Sequences<T> q, const Tensor<const T> dout,
                                                                           const float* __restrict__ dlast,
                                                                           const float* __restrict__ saved, const Tensor<T> dgates,
                                                                           const Tensor<T> dinputs, float* __restrict__ dstate,
                                                                           const Chain chain)
{
    __shared__ TileLds<V> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t block;
    const int32_t k = take_ticket<V>(chain, lds, (int32_t)((q.threads + 63) / 64), block);
    const int64_t thread = (int64_t)block * 64 + lane;
    const bool on = thread < q.threads;
    const Place<T, V> at(on ? thread : 0, q.vectors, q.channels);
    const int64_t t = (int64_t)(chain.count - 1 - k) * tile_steps(V) + (tile_waves(V) - 1 - wave) * kSteps;
    const int n = (int)max((int64_t)0, min((int64_t)kSteps, q.steps - t));
    float m[kSteps][V], d[kSteps][V], first[V], c[V];
    Vec<T, V> dys[kSteps];
    uint32_t resets;
    Maps<V> f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        f.v[v] = Map{1.0f, 0.0f};
        first[v] = dlast && on ? dlast[at.flat + v] : 0.0f;
    }
    {
        Vec<T, V> gs[kSteps], xs[kSteps];
        load_steps<T, V>(at.in(q.gates) + t * q.gates.step, q.gates.step, n, gs);
        load_steps<T, V>(at.in(q.inputs) + t * q.inputs.step, q.inputs.step, n, xs);
        load_steps<T, V>(at.in(dout) + t * dout.step, dout.step, n, dys);
        resets = load_resets<kResets, kSteps>(at.flags(q.resets) + t * q.resets.step, q.resets.step, n, q.one);
        float h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = 0.0f;
        if (on && n > 0) {
            const Vec<float, V> s = load<float, V>(saved + (t / kSteps) * q.states + at.flat);
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = s.v[v];
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float x = (float)xs[i].v[v];
                float a, b;
                m[i][v] = gate_of<T>((float)gs[i].v[v]);
                gate_parts(m[i][v], a, b);
                if (kResets && (resets >> i & 1u)) h[v] = 0.0f;
                d[i][v] = h[v] - x;
                h[v] = fmaf(a, h[v], b * x);
                hold(m[i][v]);
                hold(d[i][v]);
            }
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        const int i = kSteps - 1 - j;
        if (i >= n) continue;
        hold(dys[i]);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float a, b;
            gate_parts(m[i][v], a, b);
            const bool reset = kResets && (resets >> i & 1u);
            f.v[v].H = reset ? 0.0f : a * ((float)dys[i].v[v] + f.v[v].H);
            f.v[v].P = reset ? -0.0f : a * f.v[v].P;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) f.v[v].P = kept(f.v[v].P);
    state_before<V>(chain, lds, q.threads, thread, on, k, wave, f, first, c);
    if (!on) return;
    T* dg = at.in(dgates) + t * dgates.step;
    T* dx = at.in(dinputs) + t * dinputs.step;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        const int i = kSteps - 1 - j;
        if (i >= n) continue;
        hold(dys[i]);
        Vec<T, V> og, ox;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float a, b;
            gate_parts(m[i][v], a, b);
            const float G = (float)dys[i].v[v] + c[v], bG = b * G;
            ox.v[v] = (T)bG;
            og.v[v] = (T)(a * bG * d[i][v]);
            c[v] = kResets && (resets >> i & 1u) ? 0.0f : a * G;
        }
        store<T, V>(dg + i * dgates.step, og);
        store<T, V>(dx + i * dinputs.step, ox);
    }
    if (dstate && t == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) dstate[at.flat + v] = c[v];
    }
}

// ---------------------------------------------------------------------------
// many channels: a thread walks through all steps of its own
// ---------------------------------------------------------------------------

template <class T, int V, bool kResets>
__global__ __launch_bounds__(256) void scan_kernel(const Sequences<T> q, const Tensor<T> out, float* __restrict__ last,
                                                   float* __restrict__ saved)
{
    const int64_t thread = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (thread >= q.threads) return;
    const Place<T, V> at(thread, q.vectors, q.channels);
    const T* g = at.in(q.gates);
    const T* x = at.in(q.inputs);
    const uint8_t* r = at.flags(q.resets);
    T* y = at.in(out);
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = q.state ? q.state[at.flat + v] : 0.0f;
    auto steps = [&](int64_t t, int n) {
        Vec<T, V> gs[kSteps], xs[kSteps];
        load_steps<T, V>(g + t * q.gates.step, q.gates.step, n, gs);
        load_steps<T, V>(x + t * q.inputs.step, q.inputs.step, n, xs);
        const uint32_t resets = load_resets<kResets, kSteps>(r + t * q.resets.step, q.resets.step, n, q.one);
        if (saved) {
            Vec<float, V> s;
#pragma unroll
            for (int v = 0; v < V; ++v) s.v[v] = h[v];
            store<float, V>(saved + (t / kSteps) * q.states + at.flat, s);
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (i >= n) continue;
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float a, b;
                gate_parts(gate_of<T>((float)gs[i].v[v]), a, b);
                const float add = b * (float)xs[i].v[v];
                h[v] = kResets && (resets >> i & 1u) ? add : fmaf(a, h[v], add);
                o.v[v] = (T)h[v];
            }
            store<T, V>(y + (t + i) * out.step, o);
        }
    };
    int64_t t = 0;
    for (; t + kSteps <= q.steps; t += kSteps) steps(t, kSteps);
    if (t < q.steps) steps(t, (int)(q.steps - t));
    if (last) {
#pragma unroll
        for (int v = 0; v < V; ++v) last[at.flat + v] = h[v];
    }
}

template <class T, int V, bool kResets>
__global__ __launch_bounds__(256, 4) void scan_gradient_kernel(const Sequences<T> q, const Tensor<const T> dout,
                                                            const float* __restrict__ dlast, const float* __restrict__ saved,
                                                            const Tensor<T> dgates, const Tensor<T> dinputs,
                                                            float* __restrict__ dstate)
{
    const int64_t thread = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (thread >= q.threads) return;
    const Place<T, V> at(thread, q.vectors, q.channels);
    const T* g = at.in(q.gates);
    const T* x = at.in(q.inputs);
    const T* dy = at.in(dout);
    const uint8_t* r = at.flags(q.resets);
    T* dg = at.in(dgates);
    T* dx = at.in(dinputs);
    float c[V];
#pragma unroll
    for (int v = 0; v < V; ++v) c[v] = dlast ? dlast[at.flat + v] : 0.0f;
    auto steps = [&](int64_t t, int n) {
        Vec<T, V> gs[kSteps], xs[kSteps], dys[kSteps];
        load_steps<T, V>(g + t * q.gates.step, q.gates.step, n, gs);
        load_steps<T, V>(x + t * q.inputs.step, q.inputs.step, n, xs);
        load_steps<T, V>(dy + t * dout.step, dout.step, n, dys);
        const uint32_t resets = load_resets<kResets, kSteps>(r + t * q.resets.step, q.resets.step, n, q.one);
        const Vec<float, V> s = load<float, V>(saved + (t / kSteps) * q.states + at.flat);
        float h[V], m[kSteps][V], d[kSteps][V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = s.v[v];
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float xi = (float)xs[i].v[v];
                float a, b;
                m[i][v] = gate_of<T>((float)gs[i].v[v]);
                gate_parts(m[i][v], a, b);
                if (kResets && (resets >> i & 1u)) h[v] = 0.0f;
                d[i][v] = h[v] - xi;
                h[v] = fmaf(a, h[v], b * xi);
                hold(m[i][v]);
                hold(d[i][v]);
            }
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const int i = kSteps - 1 - j;
            if (i >= n) continue;
            hold(dys[i]);
            Vec<T, V> og, ox;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float a, b;
                gate_parts(m[i][v], a, b);
                const float G = (float)dys[i].v[v] + c[v], bG = b * G;
                ox.v[v] = (T)bG;
                og.v[v] = (T)(a * bG * d[i][v]);
                c[v] = kResets && (resets >> i & 1u) ? 0.0f : a * G;
            }
            store<T, V>(dg + (t + i) * dgates.step, og);
            store<T, V>(dx + (t + i) * dinputs.step, ox);
        }
    };
    int64_t t = q.steps;
    if (t % kSteps) {
        t -= t % kSteps;
        steps(t, (int)(q.steps - t));
    }
    for (; t > 0; t -= kSteps) steps(t - kSteps, kSteps);
    if (dstate) {
#pragma unroll
        for (int v = 0; v < V; ++v) dstate[at.flat + v] = c[v];
    }
}

// One step in place: as many channels a thread as 16 bytes hold, at any address.  (The last
// ones of a sequence one by one: a state is read before it is replaced, so no two threads
// may hold a channel.  out and state may be a thread's own operands: no __restrict__.)
template <class T>
__global__ __launch_bounds__(256) void step_kernel(const Sequences<T> q, T* out, int64_t out_batch, float* state)
{
    constexpr int V = 16 / sizeof(T);
    const int64_t thread = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (thread >= q.threads) return;
    const Place<T, 1> at(thread, q.vectors, q.vectors);   // (at.c: the vector)
    const int32_t c = at.c * V, n = min(V, q.channels - c);
    const T* gates = q.gates.data + at.b * q.gates.batch + c;
    const T* inputs = q.inputs.data + at.b * q.inputs.batch + c;
    float* states = state + at.b * q.channels + c;
    T* to = out + at.b * out_batch + c;
    Vec<T, V> g, x, o;
    Vec<float, V> h;
    if (n == V) {
        g = load<T, V>(gates);
        x = load<T, V>(inputs);
        h = load<float, V>(states);
    } else {
        g = x = Vec<T, V>{};
        h = Vec<float, V>{};
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v < n) g.v[v] = gates[v], x.v[v] = inputs[v], h.v[v] = states[v];
    }
    const bool reset = q.resets.data && q.resets.data[at.b * q.resets.batch];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float a, b;
        gate_parts(gate_of<T>((float)g.v[v]), a, b);
        const float add = b * (float)x.v[v];
        h.v[v] = reset ? add : fmaf(a, h.v[v], add);
        o.v[v] = (T)h.v[v];
    }
    if (n == V) {
        store<float, V>(states, h);
        store<T, V>(to, o);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v < n) states[v] = h.v[v], to[v] = o.v[v];
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

size_t size_of(int32_t t) { return t == PICTURA_F32 ? 4 : 2; }

// Waves from which on every thread walks through all steps.  Walking against tiles, us (512
// steps):
//     bf16      512 waves forward 139 and 97, gradient 372 and 151 (64 M elements)
//             1,024 waves 82 and 102, 151 and 157 (of 2,048 steps 329 and 357, 604 and 549)
//             1,600 waves 136 and 141, 265 and 226
//     fp32      512 waves 42 and 41, 83 and 75
//             1,024 waves 80 and 86, 130 and 132 (of 2,048 steps 316 and 324, 522 and 499)
//             4,096 waves 309 and 299, 514 and 467
constexpr int64_t kManyWaves = 1024;
constexpr int64_t many_back(int vec) { return vec == 2 ? 2048 : 8192; }

// Channels of a thread: two of 16 bits, as one load.
int32_t vector_of(const pictura_sequences& q) { return q.dtype != PICTURA_F32 && q.channels > 1 ? 2 : 1; }

// Channels of a thread, and the tiles that the steps are cut into (0: not cut).
struct Shape {
    int32_t vec, tiles;
    int64_t threads;
};

int64_t vectors_of(int32_t channels, int32_t vec) { return ((int64_t)channels + vec - 1) / vec; }

Shape shape_of(const pictura_sequences& q, int32_t vec, bool back)
{
    Shape s{vec, 0, q.batch * vectors_of(q.channels, vec)};
    const int64_t waves = (s.threads + 63) / 64, tile = tile_steps(vec), tiles = (q.steps + tile - 1) / tile;
    // (a launch has fewer than 2^32 threads)
    if (waves < (back ? many_back(vec) : kManyWaves) && q.steps >= 2 * tile && waves * tiles <= 1 << 21) s.tiles = (int32_t)tiles;
    return s;
}

int64_t chain_words(const Shape& s) { return (int64_t)(s.tiles + (s.tiles + kGroup - 1) / kGroup) * s.threads * s.vec; }

uint64_t workspace_bytes_of(const pictura_sequences& q)
{
    return 256 + sizeof(Word) * (uint64_t)chain_words(shape_of(q, vector_of(q), true));
}

constexpr int64_t kMostChannels = (1ll << 31) - 1;   // of all sequences together

bool sizes_ok(const pictura_sequences* q)
{
    return q && (q->dtype == PICTURA_F32 || q->dtype == PICTURA_BF16 || q->dtype == PICTURA_F16) && q->batch >= 0 &&
           q->steps >= 0 && q->steps <= 0x7FFFFFFFll && q->channels >= 1 && q->batch <= kMostChannels / q->channels;
}

bool strides_ok(int64_t batch, int64_t step) { return batch >= 0 && step >= 0; }

// Written tensors: no two elements at one place.
bool apart(const pictura_sequences& q, int64_t batch, int64_t step)
{
    if (!strides_ok(batch, step)) return false;
    const bool many = q.batch > 1, more = q.steps > 1;
    if ((many && batch < q.channels) || (more && step < q.channels)) return false;
    return !many || !more || batch / step >= q.steps || step / batch >= q.batch;   // one spans all of the other
}

// What a step writes is either a thread's own operands or apart from all that is read: threads
// run in any order.
bool step_apart(const pictura_sequences& q, const void* out, int64_t out_batch, const float* state)
{
    const int64_t e = (int64_t)size_of(q.dtype);
    auto rows = [&](const void* p, int64_t batch) { return region(p, q.batch, q.channels * e, batch * e); };
    const Region y = rows(out, out_batch), h = region(state, q.batch, q.channels * 4ll, q.channels * 4ll);
    for (const Region& r : {rows(q.gates, q.gates_batch), rows(q.inputs, q.inputs_batch)})
        if ((overlap(r, y) && !same(r, y)) || (overlap(r, h) && !same(r, h))) return false;
    const Region flags = region(q.resets, q.batch, 1, q.resets_batch);
    return !(overlap(y, h) && !same(y, h)) && !overlap(flags, y) && !overlap(flags, h);
}

bool inputs_ok(const pictura_sequences& q)
{
    const size_t e = size_of(q.dtype);
    return q.gates && q.inputs && aligned(q.gates, e) && aligned(q.inputs, e) && aligned(q.state, 4) &&
           strides_ok(q.gates_batch, q.gates_step) && strides_ok(q.inputs_batch, q.inputs_step) &&
           strides_ok(q.resets_batch, q.resets_step);
}

pictura_status launched() { return hipGetLastError() == hipSuccess ? PICTURA_OK : PICTURA_EDEVICE; }

template <class T>
Sequences<T> sequences_of(const pictura_sequences& q, const Shape& s)
{
    const int64_t vectors = vectors_of(q.channels, s.vec);
    return Sequences<T>{{(const T*)q.gates, q.gates_batch, q.gates_step}, {(const T*)q.inputs, q.inputs_batch, q.inputs_step},
                        q.state, {q.resets, q.resets_batch, q.resets_step}, s.threads, q.steps,
                        q.batch * q.channels, q.channels, (int32_t)vectors, vectors % 64 == 0};
}

Chain chain_of(void* workspace, const Shape& s)
{
    Word* words = (Word*)((char*)workspace + 256);
    return Chain{(uint32_t*)workspace, words, words + (int64_t)s.tiles * s.threads * s.vec, chain_words(s), s.tiles};
}

void clear(const Chain& c, hipStream_t st)
{
    hipLaunchKernelGGL(chain_kernel, dim3((unsigned)((c.words + 255) / 256)), dim3(256), 0, st, c);
}

// go(T{}, constant V, constant whether there are resets)
template <bool B>
struct Bool {
    static constexpr bool value = B;
};
template <int N>
struct Int {
    static constexpr int value = N;
};

template <class F>
void with_kinds(const pictura_sequences& q, int32_t vec, F go)
{
    auto resets = [&](auto t, auto v) {
        if (q.resets) go(t, v, Bool<true>{});
        else go(t, v, Bool<false>{});
    };
    auto typed = [&](auto t) {
        if constexpr (sizeof(t) == 2)
            if (vec == 2) return resets(t, Int<2>{});
        resets(t, Int<1>{});
    };
    if (q.dtype == PICTURA_F32) typed(float{});
    else if (q.dtype == PICTURA_BF16) typed((__bf16)0.0f);
    else typed((_Float16)0.0f);
}

dim3 grid_of(const Shape& s)
{
    return s.tiles ? dim3((unsigned)((s.threads + 63) / 64 * s.tiles)) : dim3((unsigned)((s.threads + 255) / 256));
}

}  // namespace
}  // namespace pictura

using namespace pictura;

extern "C" {

pictura_status pictura_gated_scan_workspace(const pictura_sequences* q, uint64_t* bytes)
{
    if (!sizes_ok(q) || !bytes) return PICTURA_EINVAL;
    *bytes = workspace_bytes_of(*q);
    return PICTURA_OK;
}

pictura_status pictura_gated_scan(const pictura_sequences* q, void* out, int64_t out_batch, int64_t out_step,
                                  float* last_state, float* saved, void* workspace, uint64_t workspace_bytes, void* stream)
{
    if (!sizes_ok(q)) return PICTURA_EINVAL;
    if (q->batch == 0) return PICTURA_OK;
    const size_t e = size_of(q->dtype);
    if (!aligned(last_state, 4) || !aligned(q->state, 4)) return PICTURA_EINVAL;
    if (q->steps == 0 && !last_state) return PICTURA_OK;   // (nothing to write)
    if (q->steps > 0) {
        if (!inputs_ok(*q) || !out || !aligned(out, e) || !apart(*q, out_batch, out_step) || !aligned(saved, 4))
            return PICTURA_EINVAL;
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < workspace_bytes_of(*q)) return PICTURA_EINVAL;
    }
    const Shape s = shape_of(*q, vector_of(*q), false);
    hipStream_t st = (hipStream_t)stream;
    with_kinds(*q, s.vec, [&](auto t, auto v, auto resets) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        constexpr bool R = decltype(resets)::value;
        const Sequences<T> seq = sequences_of<T>(*q, s);
        const Tensor<T> y{(T*)out, out_batch, out_step};
        if (s.tiles) {
            const Chain c = chain_of(workspace, s);
            clear(c, st);
            hipLaunchKernelGGL((tile_kernel<T, V, R>), grid_of(s), dim3(tile_waves(V) * 64), 0, st, seq, y, last_state, saved, c);
        } else {
            hipLaunchKernelGGL((scan_kernel<T, V, R>), grid_of(s), dim3(256), 0, st, seq, y, last_state, saved);
        }
    });
    return launched();
}

pictura_status pictura_gated_scan_gradient(const pictura_sequences* q, const float* saved, const void* dout, int64_t dout_batch,
                                           int64_t dout_step, const float* dlast, void* dgates, int64_t dgates_batch,
                                           int64_t dgates_step, void* dinputs, int64_t dinputs_batch, int64_t dinputs_step,
                                           float* dstate, void* workspace, uint64_t workspace_bytes, void* stream)
{
    if (!sizes_ok(q)) return PICTURA_EINVAL;
    if (q->batch == 0) return PICTURA_OK;
    const size_t e = size_of(q->dtype);
    if (!aligned(dlast, 4) || !aligned(dstate, 4)) return PICTURA_EINVAL;
    if (q->steps == 0 && !dstate) return PICTURA_OK;   // (nothing to write)
    if (q->steps > 0) {
        if (!inputs_ok(*q) || !saved || !aligned(saved, 4) || !dout || !aligned(dout, e) || !strides_ok(dout_batch, dout_step))
            return PICTURA_EINVAL;
        if (!dgates || !dinputs || !aligned(dgates, e) || !aligned(dinputs, e) || !apart(*q, dgates_batch, dgates_step) ||
            !apart(*q, dinputs_batch, dinputs_step))
            return PICTURA_EINVAL;
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < workspace_bytes_of(*q)) return PICTURA_EINVAL;
    }
    const Shape s = shape_of(*q, vector_of(*q), true);
    hipStream_t st = (hipStream_t)stream;
    with_kinds(*q, s.vec, [&](auto t, auto v, auto resets) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        constexpr bool R = decltype(resets)::value;
        const Sequences<T> seq = sequences_of<T>(*q, s);
        const Tensor<const T> dy{(const T*)dout, dout_batch, dout_step};
        const Tensor<T> dg{(T*)dgates, dgates_batch, dgates_step}, dx{(T*)dinputs, dinputs_batch, dinputs_step};
        if (s.tiles) {
            const Chain c = chain_of(workspace, s);
            clear(c, st);
            hipLaunchKernelGGL((tile_gradient_kernel<T, V, R>), grid_of(s), dim3(tile_waves(V) * 64), 0, st, seq, dy, dlast, saved, dg,
                               dx, dstate, c);
        } else {
            hipLaunchKernelGGL((scan_gradient_kernel<T, V, R>), grid_of(s), dim3(256), 0, st, seq, dy, dlast, saved, dg, dx, dstate);
        }
    });
    return launched();
}

pictura_status pictura_gated_step(const pictura_sequences* q, void* out, int64_t out_batch, float* state, void* stream)
{
    if (!sizes_ok(q) || q->steps != 1) return PICTURA_EINVAL;
    if (q->batch == 0) return PICTURA_OK;
    const size_t e = size_of(q->dtype);
    if (!inputs_ok(*q) || !out || !aligned(out, e) || !apart(*q, out_batch, 0) || !state || !aligned(state, 4)) return PICTURA_EINVAL;
    if (!step_apart(*q, out, out_batch, state)) return PICTURA_EINVAL;
    auto go = [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / sizeof(T);
        const Shape s{V, 0, q->batch * vectors_of(q->channels, V)};
        hipLaunchKernelGGL(step_kernel<T>, dim3((unsigned)((s.threads + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                           sequences_of<T>(*q, s), (T*)out, out_batch, state);
    };
    if (q->dtype == PICTURA_F32) go(float{});
    else if (q->dtype == PICTURA_BF16) go((__bf16)0.0f);
    else go((_Float16)0.0f);
    return launched();
}

}  // extern "C"
