// Root-mean-square norm of rows with the residual's addition, its gradient, and the
// norm with an output in 8 bits.
//
//     s = x + r,  q = 1 / sqrt(mean(s^2) + eps),  y = (s q) w
//     k = dy w,  ds = q (k - (s q) mean(k s q)) + dsum,  dw = sum over rows of dy (s q)
//
// A row is held in the registers of a group of lanes, a wave or a workgroup, and read once.
// Vectors of 16 bytes are loaded at any address; where a row's length is no multiple of them
// the last one covers the row's end, and so repeats some elements of the one before
// (both lanes write the same values there; sums skip the second ones).
//
// The mean is summed in 64 bits and q rounded once, so that it hangs neither on how a row
// is split nor on the order of a sum; the codes of an 8-bit output, which change by a whole
// step at a border, then repeat to the bit.
//
// Bound by memory.  Measured (one MI355X, large copies at 5,150 GB/s): 262,144 rows of 512 in
// bf16 with residual forward 181 us, gradient 203 and the sums of dw 7 (1,074 MB each: 5.9 and
// 5.3 TB/s, some of it from the caches); 65,536 of 512 to e4m3 51 us, their values 25; 4,095
// of 8,197 in fp32 98, 110 and 7 us (537 MB each: 5.5 and 4.9 TB/s).  In rows of more than 16,384
// elements the gradient spills 110 to 160 registers, of more than 32,768 some 520 to 610 (and the
// forward 60 to 80): in bf16 2,048 of 32,768 forward 118 us, gradient 319, 1,024 of 65,536 230 and
// 630; in fp32 1,024 of 32,768 108 and 280, 512 of 65,536 200 and 476.
#include <cmath>

#include "pictura.h"
#include "pictura_lanes.h"
#include "pictura_overlap.h"

#pragma clang fp contract(off)

namespace pictura {
namespace {

template <class T>
struct Rows {
    const T* x;
    const T* residual;
    const void* weight;   // T or float
    int64_t x_stride, residual_stride, rows;
    int32_t width;
    float eps;
};

// Sum over the G lanes of a group, the same in each.
template <int G, class V>
__device__ __forceinline__ V group_sum(V x)
{
    x = x + lanes<0xB1, 0xf>((V)0, x);                      // neighbours, pairs, fours, eights
    if constexpr (G > 2) x = x + lanes<0x4E, 0xf>((V)0, x);
    if constexpr (G > 4) x = x + lanes<0x141, 0xf>((V)0, x);
    if constexpr (G > 8) x = x + lanes<0x140, 0xf>((V)0, x);
    if constexpr (G > 16) x = x + __shfl_xor(x, 16);
    if constexpr (G > 32) x = x + __shfl_xor(x, 32);
    return x;
}

template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t x)
{
    x = max(x, lanes<0xB1, 0xf>(0u, x));
    if constexpr (G > 2) x = max(x, lanes<0x4E, 0xf>(0u, x));
    if constexpr (G > 4) x = max(x, lanes<0x141, 0xf>(0u, x));
    if constexpr (G > 8) x = max(x, lanes<0x140, 0xf>(0u, x));
    if constexpr (G > 16) x = max(x, (uint32_t)__shfl_xor((int)x, 16));
    if constexpr (G > 32) x = max(x, (uint32_t)__shfl_xor((int)x, 32));
    return x;
}

// The lanes that hold a row: G of a wave (NW = 1; 64 / G rows a wave, four waves a
// workgroup), or a workgroup of NW waves (G = 64).
template <int G_, int NW_>
struct Team {
    static constexpr int G = G_, NW = NW_, kLanes = G * NW;
    static constexpr int kThreads = NW == 1 ? 256 : NW * 64;
    static constexpr int kRows = kThreads / kLanes;   // rows of a workgroup at a time
    __device__ __forceinline__ static int member() { return threadIdx.x % kLanes; }
    __device__ __forceinline__ static int row() { return threadIdx.x / kLanes; }
    template <class V>
    __device__ __forceinline__ static V sum(V x, V* lds)
    {
        x = group_sum<G>(x);
        if constexpr (NW > 1) {
            __syncthreads();   // (lds may still be read from before)
            if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
            __syncthreads();
            x = group_sum<NW>(lds[threadIdx.x & (NW - 1)]);
        }
        return x;
    }
    __device__ __forceinline__ static uint32_t most(uint32_t x, uint32_t* lds)
    {
        x = group_max<G>(x);
        if constexpr (NW > 1) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
            __syncthreads();
            x = group_max<NW>(lds[threadIdx.x & (NW - 1)]);
        }
        return x;
    }
};

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

// Where the vectors of a lane stand in a row of C elements, the j-th of NV: its first
// element, whether there is one, and how many of its first elements an earlier one holds.
template <int V, int kLanes>
struct Span {
    int first, again;
    bool on;
    __device__ __forceinline__ Span(int member, int j, int C)
    {
        const int at = (j * kLanes + member) * V;
        on = at < C;
        first = at + V <= C ? at : C - V;   // (C is V or more)
        again = on ? at - first : 0;
    }
};

__device__ __forceinline__ float factor(double sum, int32_t width, float eps)
{
    return (float)(1.0 / __builtin_sqrt(sum / (double)width + (double)eps));
}

// out: T, or 8-bit codes with a scale for each row.  sum and out may be the rows that are read (all of
// a row is before any of it is written): no __restrict__.
struct Codes {
    void* codes;
    int64_t stride;
    float* scales;
    int32_t kind;
};

template <class T, class W, int V, int NV, class Tm, bool kCodes>
__global__ __launch_bounds__(Tm::kThreads) void norm_kernel(const Rows<T> R, T* sum, int64_t sum_stride,
                                                            T* out, int64_t out_stride,
                                                            float* __restrict__ factors, const Codes codes)
{
    __shared__ double ldsd[Tm::NW];
    __shared__ uint32_t ldsu[Tm::NW];
    const int C = R.width;
    // (all lanes of a row together; more than one row only beyond what a launch holds)
    for (int64_t n = (int64_t)blockIdx.x * Tm::kRows + Tm::row(); n < R.rows; n += (int64_t)gridDim.x * Tm::kRows) {
        const T* x = R.x + n * R.x_stride;
        const T* r = R.residual + n * R.residual_stride;
        float s[NV][V];
        Vec<T, V> xs[NV], rs[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Span<V, Tm::kLanes> at(Tm::member(), j, C);
            xs[j] = rs[j] = Vec<T, V>{};
            if (at.on) xs[j] = load<T, V>(x + at.first);
            if (at.on && R.residual) rs[j] = load<T, V>(r + at.first);
        }
        double total = 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Span<V, Tm::kLanes> at(Tm::member(), j, C);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[j][v] = (float)xs[j].v[v];
                if (R.residual) s[j][v] = (float)(xs[j].v[v] = (T)(s[j][v] + (float)rs[j].v[v]));
                const double d = v >= at.again ? (double)s[j][v] : 0.0;
                total = fma(d, d, total);
            }
        }
        total = Tm::sum(total, ldsd);
        const float q = factor(total, C, R.eps);
        if (sum) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const Span<V, Tm::kLanes> at(Tm::member(), j, C);
                if (at.on) store<T, V>(sum + n * sum_stride + at.first, xs[j]);
            }
        }
        if (factors && Tm::member() == 0) factors[n] = q;
        uint32_t most = 0;   // bits of the largest magnitude: a NaN is the largest of all
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Span<V, Tm::kLanes> at(Tm::member(), j, C);
            if (!at.on) continue;
            const Vec<W, V> w = load<W, V>((const W*)R.weight + at.first);
            Vec<T, V> y;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float z = (s[j][v] * q) * (float)w.v[v];
                if constexpr (kCodes) {
                    s[j][v] = z;
                    most = max(most, __float_as_uint(fabsf(z)));
                } else {
                    y.v[v] = (T)z;
                }
            }
            if constexpr (!kCodes) store<T, V>(out + n * out_stride + at.first, y);
        }
        if constexpr (kCodes) {
            const bool e4m3 = codes.kind == PICTURA_E4M3;
            const float level = e4m3 ? 448.0f : 127.0f, top = __uint_as_float(Tm::most(most, ldsu));
            const bool none = top < 0x1p-100f;   // (level / top would leave fp32's range)
            const float up = none ? 0.0f : level * (1.0f / top);
            if (Tm::member() == 0) codes.scales[n] = none ? 0.0f : top / level;
            uint8_t* to = (uint8_t*)codes.codes + n * codes.stride;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const Span<V, Tm::kLanes> at(Tm::member(), j, C);
                if (!at.on) continue;
                Vec<uint8_t, V> c;
                if (e4m3) {
#pragma unroll
                    for (int v = 0; v < V; v += 2) {
                        const int two = __builtin_amdgcn_cvt_pk_fp8_f32(s[j][v] * up, v + 1 < V ? s[j][v + 1 < V ? v + 1 : v] * up : 0.0f, 0, false);
                        c.v[v] = (uint8_t)two;
                        if (v + 1 < V) c.v[v + 1 < V ? v + 1 : v] = (uint8_t)(two >> 8);
                    }
                } else {
#pragma unroll
                    for (int v = 0; v < V; ++v) c.v[v] = (uint8_t)(int8_t)(int)rintf(s[j][v] * up);
                }
                store<uint8_t, V>(to + at.first, c);
            }
        }
    }
}

// What codes stand for, four a thread at any address, the last ones of a row one by one.
__device__ __forceinline__ float value_of(uint8_t code, int32_t kind)
{
    return kind == PICTURA_E4M3 ? __builtin_amdgcn_cvt_f32_fp8((int)code, 0) : (float)(int8_t)code;
}

static __global__ __launch_bounds__(256) void values_kernel(const uint8_t* __restrict__ codes, int64_t stride,
                                                            const float* __restrict__ scales, int32_t kind, int64_t rows,
                                                            int32_t width, float* __restrict__ out, int64_t out_stride)
{
    constexpr int V = 4;
    const int32_t per = (width + V - 1) / V;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * per) return;
    int64_t n;
    int32_t c;
    if (i >> 32 == 0) {
        n = (uint32_t)i / (uint32_t)per;
        c = (int32_t)((uint32_t)i % (uint32_t)per) * V;
    } else {
        n = i / per;
        c = (int32_t)(i % per) * V;
    }
    const float scale = scales[n];
    codes += n * stride + c;
    out += n * out_stride + c;
    if (c + V <= width) {
        const Vec<uint8_t, V> q = load<uint8_t, V>(codes);
        Vec<float, V> y;
#pragma unroll
        for (int v = 0; v < V; ++v) y.v[v] = value_of(q.v[v], kind) * scale;
        store<float, V>(out, y);
    } else {
        for (int v = 0; v < width - c; ++v) out[v] = value_of(codes[v], kind) * scale;
    }
}

template <class T>
struct Gradient {
    const T* s;
    const T* dout;
    const T* dsum;   // or null
    const float* factors;
    const void* weight;
    T* dx;
    float* part;     // [parts][width]: sums over the rows of each workgroup
    int64_t s_stride, dout_stride, dsum_stride, dx_stride, rows;
    int32_t width;
};

// Teams take rows in turn, one workgroup's the same distance apart, and keep the sums of
// dy (s q) of their columns in registers: in fp32, as fp64 would take twice the
// registers.  A team adds up some 16 rows (4,095 of 8,197 in fp32: dw is off by 9e-8, and by 5e-8
// if summed in 64 bits) to 32 (262,144 of 512), the workgroups' sums are added up in fp64.
template <class T, class W, int V, int NV, class Tm>
__global__ __launch_bounds__(Tm::kThreads) void norm_gradient_kernel(const Gradient<T> R)
{
    __shared__ float lds[Tm::NW];
    const int C = R.width;
    const float inverse = 1.0f / (float)C;
    const int64_t first = (int64_t)blockIdx.x * Tm::kRows + Tm::row(), step = (int64_t)gridDim.x * Tm::kRows;
    float dw[NV][V] = {};
    for (int64_t n = first; n < R.rows; n += step) {
        Vec<T, V> ss[NV], dys[NV], ds[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Span<V, Tm::kLanes> at(Tm::member(), j, C);
            ss[j] = dys[j] = ds[j] = Vec<T, V>{};
            if (at.on) {
                ss[j] = load<T, V>(R.s + n * R.s_stride + at.first);
                dys[j] = load<T, V>(R.dout + n * R.dout_stride + at.first);
                if (R.dsum) ds[j] = load<T, V>(R.dsum + n * R.dsum_stride + at.first);
            }
        }
        const float q = R.factors[n];
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Span<V, Tm::kLanes> at(Tm::member(), j, C);
            Vec<W, V> w{};
            if (at.on) w = load<W, V>((const W*)R.weight + at.first);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float u = (float)ss[j].v[v] * q, dy = (float)dys[j].v[v], t = dy * u;
                if (v >= at.again) dot = fmaf(t, (float)w.v[v], dot);
                dw[j][v] += t;
            }
        }
        dot = Tm::sum(dot, lds) * inverse;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Span<V, Tm::kLanes> at(Tm::member(), j, C);
            if (!at.on) continue;
            const Vec<W, V> w = load<W, V>((const W*)R.weight + at.first);
            Vec<T, V> o;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float u = (float)ss[j].v[v] * q, k = (float)dys[j].v[v] * (float)w.v[v];
                o.v[v] = (T)fmaf(q, fmaf(-u, dot, k), (float)ds[j].v[v]);
            }
            store<T, V>(R.dx + n * R.dx_stride + at.first, o);
        }
    }
    float* part = R.part + (int64_t)blockIdx.x * C;
    if constexpr (Tm::kRows == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const Span<V, Tm::kLanes> at(Tm::member(), j, C);
            if (!at.on) continue;
            Vec<float, V> o;
#pragma unroll
            for (int v = 0; v < V; ++v) o.v[v] = dw[j][v];
            store<float, V>(part + at.first, o);
        }
    } else {   // the workgroup's teams are added up, in their order
        constexpr int kSlots = Tm::kLanes * V;
        __shared__ float all[Tm::kRows][kSlots + 1];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v) all[Tm::row()][Tm::member() * V + v] = dw[j][v];
            __syncthreads();
            for (int i = threadIdx.x; i < kSlots; i += Tm::kThreads) {
                float x = 0.0f;
                for (int k = 0; k < Tm::kRows; ++k) x += all[k][i];
                const Span<V, Tm::kLanes> at(i / V, j, C);
                if (at.on) part[at.first + i % V] = x;   // (what two vectors hold is the same in both)
            }
        }
    }
}

// Sums of the parts, 16 columns to a workgroup of 64 rows of threads, in a fixed order.
constexpr int kColumns = 16, kDeep = 64;
template <class W>
__global__ __launch_bounds__(kColumns * kDeep) void weight_gradient_kernel(const float* __restrict__ part, int32_t parts,
                                                                           int32_t width, W* __restrict__ dweight)
{
    __shared__ double lds[kDeep][kColumns + 1];
    const int c = threadIdx.x % kColumns, d = threadIdx.x / kColumns;
    const int column = blockIdx.x * kColumns + c;
    double x = 0.0;
    if (column < width) {
        constexpr int kAhead = 8;   // loads under way
        for (int k = d; k < parts; k += kDeep * kAhead) {
            float y[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) y[u] = k + u * kDeep < parts ? part[(int64_t)(k + u * kDeep) * width + column] : 0.0f;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) x += (double)y[u];
        }
    }
    lds[d][c] = x;
    __syncthreads();
    for (int half = kDeep / 2; half > 0; half /= 2) {
        if (d < half) lds[d][c] += lds[d + half][c];
        __syncthreads();
    }
    if (d == 0 && column < width) dweight[column] = (W)(float)lds[0][c];
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool known(int32_t t) { return t == PICTURA_F32 || t == PICTURA_BF16 || t == PICTURA_F16; }

size_t size_of(int32_t t) { return t == PICTURA_F32 ? 4 : 2; }

bool stride_ok(int64_t stride, int64_t rows, int32_t width, bool written)
{
    return rows < 2 || (written ? stride >= width : stride >= 0);
}

bool norm_ok(const pictura_norm* n)
{
    return n && known(n->dtype) && (n->weight_dtype == n->dtype || n->weight_dtype == PICTURA_F32) && n->rows >= 0 &&
           n->rows <= 0x7FFFFFFFll && n->width >= 1 && n->width <= PICTURA_MAX_NORM && n->eps >= 0.0f && std::isfinite(n->eps);
}

bool operands_ok(const pictura_norm& n)
{
    const size_t e = size_of(n.dtype);
    return n.x && aligned(n.x, e) && aligned(n.residual, e) && n.weight && aligned(n.weight, size_of(n.weight_dtype)) &&
           stride_ok(n.x_stride, n.rows, n.width, false) && stride_ok(n.residual_stride, n.rows, n.width, false);
}

bool output_ok(const void* p, int64_t stride, const pictura_norm& n, size_t e)
{
    return p && aligned(p, e) && stride_ok(stride, n.rows, n.width, true);
}

pictura_status launched() { return hipGetLastError() == hipSuccess ? PICTURA_OK : PICTURA_EDEVICE; }

template <int N>
struct Int {
    static constexpr int value = N;
};

// go(V, NV, Team): the lanes and registers of a row.  Rows shorter than a vector take
// single elements.  Two vectors a lane, so that a wave has more rows or bytes under way,
// are as good as one or better up to a wave's width (131,072 rows of 300 in bf16: forward 68
// us and 74, gradient 73 and 81; 262,144 of 512: 192 and 196, 199 and 208), except where codes
// of 16-bit rows come out and most lanes have a vector (65,536 to e4m3 with a residual, two a
// lane and one: of 400 38.1 and 37.2, 448 39.1 and 36.3, 480 40.4 and 38.5, 512 42.7 and 41.7;
// but in fp32 of 224 30.2 and 32.4, of 256 33.6 and 36.4).
// Wider rows of 16 bits take one a lane and more waves, whose registers then hold all of
// a row in fp32 (32,768 rows of 2,048 by one wave or four: forward 111 and 98 us, codes 109 and
// 97, gradient 128 and 109); fp32 rows four (32,768 of 1,024: 94 and 99, 81 and 83, 105 and 120).
template <class T, bool kCodes, class F>
void with_team(int32_t width, F go)
{
    constexpr int V = 16 / sizeof(T);
    const int vectors = (width + V - 1) / V;
    if (width < V) return go(Int<1>{}, Int<1>{}, Team<8, 1>{});
    if (vectors <= 8) return go(Int<V>{}, Int<1>{}, Team<8, 1>{});
    if (vectors <= 16) return go(Int<V>{}, Int<2>{}, Team<8, 1>{});
    if (vectors <= 32) return go(Int<V>{}, Int<2>{}, Team<16, 1>{});
    if constexpr (kCodes && V == 8)
        if (vectors > 48 && vectors <= 64) return go(Int<V>{}, Int<1>{}, Team<64, 1>{});
    if (vectors <= 64) return go(Int<V>{}, Int<2>{}, Team<32, 1>{});
    if (vectors <= 128) return go(Int<V>{}, Int<2>{}, Team<64, 1>{});
    if constexpr (V == 8) {
        if (vectors <= 256) return go(Int<V>{}, Int<1>{}, Team<64, 4>{});
        if (vectors <= 512) return go(Int<V>{}, Int<1>{}, Team<64, 8>{});
        if (vectors <= 1024) return go(Int<V>{}, Int<1>{}, Team<64, 16>{});
    } else {
        if (vectors <= 256) return go(Int<V>{}, Int<4>{}, Team<64, 1>{});
        if (vectors <= 512) return go(Int<V>{}, Int<2>{}, Team<64, 4>{});
        if (vectors <= 1024) return go(Int<V>{}, Int<4>{}, Team<64, 4>{});
    }
    if (vectors <= 2048) return go(Int<V>{}, Int<2>{}, Team<64, 16>{});
    if (vectors <= 4096) return go(Int<V>{}, Int<4>{}, Team<64, 16>{});
    if constexpr (V == 8) return go(Int<V>{}, Int<8>{}, Team<64, 16>{});
    else if (vectors <= 8192) return go(Int<V>{}, Int<8>{}, Team<64, 16>{});
    else return go(Int<V>{}, Int<16>{}, Team<64, 16>{});
}

// go(T{}, W{})
template <class F>
void with_types(const pictura_norm& n, F go)
{
    if (n.dtype == PICTURA_F32) go(float{}, float{});
    else if (n.dtype == PICTURA_BF16) {
        if (n.weight_dtype == PICTURA_F32) go((__bf16)0.0f, float{});
        else go((__bf16)0.0f, (__bf16)0.0f);
    } else {
        if (n.weight_dtype == PICTURA_F32) go((_Float16)0.0f, float{});
        else go((_Float16)0.0f, (_Float16)0.0f);
    }
}

template <class T>
Rows<T> rows_of(const pictura_norm& n)
{
    return Rows<T>{(const T*)n.x, (const T*)n.residual, n.weight, n.x_stride, n.residual_stride, n.rows, n.width, n.eps};
}

// (a launch has fewer than 2^32 threads)
template <class Tm>
unsigned blocks_for(int64_t rows)
{
    const int64_t b = (rows + Tm::kRows - 1) / Tm::kRows, most = (1ll << 31) / Tm::kThreads;
    return (unsigned)(b < most ? b : most);
}

template <bool kCodes>
void launch_norm(const pictura_norm& n, void* sum, int64_t sum_stride, void* out, int64_t out_stride, float* factors,
                 const Codes& codes, hipStream_t st)
{
    with_types(n, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        with_team<T, kCodes>(n.width, [&](auto v, auto nv, auto team) {
            using Tm = decltype(team);
            hipLaunchKernelGGL((norm_kernel<T, W, decltype(v)::value, decltype(nv)::value, Tm, kCodes>),
                               dim3(blocks_for<Tm>(n.rows)), dim3(Tm::kThreads), 0, st, rows_of<T>(n),
                               (T*)sum, sum_stride, (T*)out, out_stride, factors, codes);
        });
    });
}

// Waves of the gradient, whose workgroups leave a part of dweight each.
constexpr int64_t kWaves = 4096;

template <class Tm>
int64_t gradient_blocks(int64_t rows)
{
    const int64_t b = (rows + Tm::kRows - 1) / Tm::kRows, most = Tm::NW == 1 ? kWaves / 4 : kWaves / Tm::NW;
    return b < most ? b : most;
}

int64_t gradient_parts(const pictura_norm& n)
{
    int64_t parts = 0;
    auto count = [&](auto, auto, auto team) {
        using Tm = decltype(team);
        parts = gradient_blocks<Tm>(n.rows);
    };
    if (n.dtype == PICTURA_F32) with_team<float, false>(n.width, count);
    else with_team<_Float16, false>(n.width, count);
    return parts;
}

uint64_t gradient_bytes(const pictura_norm& n) { return 256 + (uint64_t)gradient_parts(n) * n.width * sizeof(float); }

}  // namespace
}  // namespace pictura

using namespace pictura;

extern "C" {

pictura_status pictura_rms_norm(const pictura_norm* n, void* sum, int64_t sum_stride, void* out, int64_t out_stride,
                                float* factors, void* stream)
{
    if (!norm_ok(n)) return PICTURA_EINVAL;
    if (n->rows == 0) return PICTURA_OK;
    const size_t e = size_of(n->dtype);
    if (!operands_ok(*n) || !output_ok(out, out_stride, *n, e) || (sum && !output_ok(sum, sum_stride, *n, e)) || !aligned(factors, 4))
        return PICTURA_EINVAL;
    launch_norm<false>(*n, sum, sum_stride, out, out_stride, factors, Codes{}, (hipStream_t)stream);
    return launched();
}

pictura_status pictura_rms_norm_codes(const pictura_norm* n, int32_t kind, void* sum, int64_t sum_stride, void* codes,
                                      int64_t codes_stride, float* scales, void* stream)
{
    if (!norm_ok(n) || (kind != PICTURA_INT8 && kind != PICTURA_E4M3)) return PICTURA_EINVAL;
    if (n->rows == 0) return PICTURA_OK;
    if (!operands_ok(*n) || !output_ok(codes, codes_stride, *n, 1) || !scales || !aligned(scales, 4) ||
        (sum && !output_ok(sum, sum_stride, *n, size_of(n->dtype))))
        return PICTURA_EINVAL;
    launch_norm<true>(*n, sum, sum_stride, nullptr, 0, nullptr, Codes{codes, codes_stride, scales, kind}, (hipStream_t)stream);
    return launched();
}

pictura_status pictura_row_values(const void* codes, int64_t codes_stride, const float* scales, int32_t kind, int64_t rows,
                                  int32_t width, float* out, int64_t out_stride, void* stream)
{
    if ((kind != PICTURA_INT8 && kind != PICTURA_E4M3) || rows < 0 || rows > 0x7FFFFFFFll || width < 1 || width > PICTURA_MAX_NORM)
        return PICTURA_EINVAL;
    if (rows == 0) return PICTURA_OK;
    if (!codes || !scales || !out || !aligned(scales, 4) || !aligned(out, 4) || !stride_ok(codes_stride, rows, width, false) ||
        !stride_ok(out_stride, rows, width, true))
        return PICTURA_EINVAL;
    const Region y = region(out, rows, width * 4ll, out_stride * 4);   // (threads run in any order)
    if (overlap(y, region(codes, rows, width, codes_stride)) || overlap(y, region(scales, rows, 4, 4))) return PICTURA_EINVAL;
    // (a launch has fewer than 2^32 threads)
    const int64_t per = (width + 3) / 4, part = (1ll << 31) / per;
    for (int64_t n = 0; n < rows; n += part) {
        const int64_t some = rows - n < part ? rows - n : part;
        hipLaunchKernelGGL(values_kernel, dim3((unsigned)((some * per + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                           (const uint8_t*)codes + n * codes_stride, codes_stride, scales + n, kind, some, width,
                           out + n * out_stride, out_stride);
    }
    return launched();
}

pictura_status pictura_rms_norm_gradient_workspace(const pictura_norm* n, uint64_t* bytes)
{
    if (!norm_ok(n) || !bytes) return PICTURA_EINVAL;
    *bytes = gradient_bytes(*n);
    return PICTURA_OK;
}

pictura_status pictura_rms_norm_gradient(const pictura_norm* n, const float* factors, const void* dout, int64_t dout_stride,
                                         const void* dsum, int64_t dsum_stride, void* dx, int64_t dx_stride, void* dweight,
                                         void* workspace, uint64_t workspace_bytes, void* stream)
{
    if (!norm_ok(n) || n->residual || !dweight || !aligned(dweight, size_of(n->weight_dtype))) return PICTURA_EINVAL;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < gradient_bytes(*n)) return PICTURA_EINVAL;
    const size_t e = size_of(n->dtype);
    if (n->rows > 0) {
        if (!operands_ok(*n) || !factors || !aligned(factors, 4) || !dout || !aligned(dout, e) ||
            !stride_ok(dout_stride, n->rows, n->width, false) || !output_ok(dx, dx_stride, *n, e))
            return PICTURA_EINVAL;
        if (!aligned(dsum, e) || (dsum && !stride_ok(dsum_stride, n->rows, n->width, false))) return PICTURA_EINVAL;
    }
    hipStream_t st = (hipStream_t)stream;
    const int64_t parts = gradient_parts(*n);
    with_types(*n, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        if (n->rows > 0)
            with_team<T, false>(n->width, [&](auto v, auto nv, auto team) {
                using Tm = decltype(team);
                const Gradient<T> g{(const T*)n->x, (const T*)dout, (const T*)dsum, factors, n->weight, (T*)dx, (float*)workspace,
                                    n->x_stride, dout_stride, dsum_stride, dx_stride, n->rows, n->width};
                hipLaunchKernelGGL((norm_gradient_kernel<T, W, decltype(v)::value, decltype(nv)::value, Tm>),
                                   dim3((unsigned)gradient_blocks<Tm>(n->rows)), dim3(Tm::kThreads), 0, st, g);
            });
        hipLaunchKernelGGL(weight_gradient_kernel<W>, dim3((unsigned)((n->width + kColumns - 1) / kColumns)),
                           dim3(kColumns * kDeep), 0, st, (const float*)workspace, (int32_t)parts, n->width, (W*)dweight);
    });
    return launched();
}

}  // extern "C"
