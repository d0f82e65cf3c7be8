// AdamW over many tensors at once, with moments in fp32 or in 8 bits, and the
// norm of all gradients together.
//
// The tensors' pointers travel in the kernel's arguments, up to 80 tensors to a
// launch (60 with 8-bit moments, 160 in the norm), so a step copies nothing to the device
// and can be captured in a graph, in which its step number is the captured one.  A
// workgroup takes kChunk elements of one tensor.
//
// Bound by memory: 300 tensors of 50 M fp32 weights with bf16 gradients take four
// launches of 50 to 77 us (1.3 GB at 4.9 TB/s; a large copy runs at 4.9) and 43 us for the
// norm, which has to see every gradient before the first weight moves: 316 us the
// call.  64 tensors of 128 M bf16 weights with 8-bit moments take 255 to 290 us (1.27 GB at
// 4.4 to 5.0 TB/s, 77 vector instructions for 64 weights), and their moments are decoded in
// 220 to 228 us (1.26 GB at 5.6).  A step of 29 tensors is launches and the binding, 29 us.
#include <cmath>

#include "pictura.h"
#include "pictura_internal.h"

#pragma clang fp contract(off)

namespace pictura {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;                     // elements of one workgroup
constexpr int kBlk = PICTURA_ADAMW_BLOCK;
constexpr float kLeastEps = 0x1p-40f;            // from it on the hardware's root and reciprocal serve
constexpr float kTiny = 0x1p-90f;                // below it a block's moments count as zero: 1 / scale stays finite
static_assert(kChunk % kBlk == 0, "blocks do not straddle workgroups");

// A tensor, or a part of one, of a launch.  Fewer fields, more tensors to a launch:
// the arguments of a kernel take 4 KB.
struct GradArg {
    const void* grad;
    int64_t n;
    int32_t first;      // workgroup of its first chunk
    uint8_t pt, gt;     // PICTURA_F32 ..
    uint8_t vec;        // 1: four elements at a time are aligned in every array
};

struct StepArg : GradArg {
    void* param;
    void* m;
    void* v;
};

struct Step8Arg : StepArg {
    float* ms;
    float* vs;
};

template <class Arg>
struct Args {
    static constexpr int kMost = 3840 / (int)sizeof(Arg);
    Arg t[kMost];
    int32_t count;
};

struct StepFactors {
    float b1, c1, b2, c2, rbc2, eps, keep, rate;
    const float* grad_factor;
};

// Tensor of workgroup b: the last whose first workgroup is not beyond b.
template <class A>
__device__ __forceinline__ int tensor_of(const A& a, int b)
{
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.t[mid].first <= b) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Elements of any of the types, one at a time.
__device__ __forceinline__ float load_as(const void* p, int type, int64_t i)
{
    if (type == PICTURA_F32) return ((const float*)p)[i];
    if (type == PICTURA_BF16) return (float)((const __bf16*)p)[i];
    return (float)((const _Float16*)p)[i];
}

__device__ __forceinline__ void store_as(void* p, int type, int64_t i, float x)
{
    if (type == PICTURA_F32) ((float*)p)[i] = x;
    else if (type == PICTURA_BF16) ((__bf16*)p)[i] = (__bf16)x;
    else ((_Float16*)p)[i] = (_Float16)x;
}

template <class T>
struct Four {
    T v[4];
};

// Four elements from i on: loaded as they are (so that several loads are under way
// before the first is waited for), and made fp32.
__device__ __forceinline__ u32x4 load4(const void* p, int type, int64_t i)
{
    if (type == PICTURA_F32) return *(const u32x4*)((const float*)p + i);
    const u32x2 t = *(const u32x2*)((const uint16_t*)p + i);
    return u32x4{t[0], t[1], 0u, 0u};
}

__device__ __forceinline__ void as_float(u32x4 t, int type, float* x)
{
    const u32x2 low = {t[0], t[1]};
    if (type == PICTURA_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(t[k]);
    } else if (type == PICTURA_BF16) {
        const Four<__bf16> h = __builtin_bit_cast(Four<__bf16>, low);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = (float)h.v[k];
    } else {
        const Four<_Float16> h = __builtin_bit_cast(Four<_Float16>, low);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = (float)h.v[k];
    }
}

__device__ __forceinline__ void store4(void* p, int type, int64_t i, const float* x)
{
    if (type == PICTURA_F32) {
        *(f32x4*)((float*)p + i) = f32x4{x[0], x[1], x[2], x[3]};
    } else if (type == PICTURA_BF16) {
        const Four<__bf16> h = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
        *(u32x2*)((uint16_t*)p + i) = __builtin_bit_cast(u32x2, h);
    } else {
        const Four<_Float16> h = {(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3]};
        *(u32x2*)((uint16_t*)p + i) = __builtin_bit_cast(u32x2, h);
    }
}

// m and v after the gradient g, and the parameter.  kFast: with the hardware's root
// and reciprocal (a unit off each, where the correctly rounded ones take some 25
// instructions): the 8-bit step is bound by instructions, the 32-bit one by memory.
// Both instructions take subnormal numbers for 0, so the root is wrong below 2^-63 and
// the reciprocal infinite: with eps from kLeastEps on, neither shows in m / den.
template <bool kFast>
__device__ __forceinline__ float adamw(const StepFactors& f, float p, float g, float& m, float& v)
{
    m = f.b1 * m + f.c1 * g;
    v = f.b2 * v + (f.c2 * g) * g;
    if constexpr (kFast) {
        const float den = __builtin_amdgcn_sqrtf(v) * f.rbc2 + f.eps;
        return p * f.keep - f.rate * (m * __builtin_amdgcn_rcpf(den));
    }
    const float den = sqrtf(v) * f.rbc2 + f.eps;
    return p * f.keep - f.rate * (m / den);
}

// c |c| and c^2 are whole numbers below 2^24: a value takes three roundings (four
// for v), and those of the scale are shared by its block.
__device__ __forceinline__ float m_unit(float s) { return s * (float)(1.0 / 16129.0); }

__device__ __forceinline__ float v_unit(float s) { return s * (float)(1.0 / 4228250625.0); }

__device__ __forceinline__ float m_value(int c, float unit)
{
    const float x = (float)c;
    return x * fabsf(x) * unit;
}

__device__ __forceinline__ float v_value(uint32_t c, float unit)
{
    const float x = (float)c, x2 = x * x;
    return x2 * x2 * unit;
}

// rint(kLevels a^(1/2)), or a^(1/4), of the correctly rounded roots.  The hardware's
// are a unit off, which with the product moves up to 255 steps by less than 1e-4; only
// within 2e-4 of a half (one element in 2,500) are the exact ones taken.
template <int kLevels, bool kFourth>
__device__ __forceinline__ float steps_of(float a)
{
    float y = __builtin_amdgcn_sqrtf(a);
    if (kFourth) y = __builtin_amdgcn_sqrtf(y);
    y *= (float)kLevels;
    float q = rintf(y);
    if (__builtin_expect(fabsf(y - q) > 0.4998f, 0)) {
        asm volatile("" : "+v"(a));   // (a branch: computed for all, the exact roots cost what they save)
        y = sqrtf(a);
        if (kFourth) y = sqrtf(y);
        q = rintf(y * (float)kLevels);
    }
    return q;
}

// The codes of m and v, with inv = 1 / scale (0 for a scale of zero or NaN; a
// NaN comes out as 0: its scale says it).
__device__ __forceinline__ int m_code(float m, float inv)
{
    const float q = fminf(fmaxf(steps_of<127, false>(fabsf(m) * inv), 0.0f), 127.0f);
    return m < 0.0f ? -(int)q : (int)q;
}

__device__ __forceinline__ uint32_t v_code(float v, float inv)
{
    float q = fminf(fmaxf(steps_of<255, true>(v * inv), 0.0f), 255.0f);
    if (v > 0.0f && inv > 0.0f) q = fmaxf(q, 1.0f);
    return (uint32_t)q;
}

// m and v decay towards g and g^2; p = keep p - rate m / (sqrt(v) rbc2 + eps).  26 bytes
// a weight at fp32 with a bf16 gradient, read and written once; four neighbours to a
// thread where the addresses allow 16-byte accesses.
__global__ __launch_bounds__(kThreads) void adamw32_kernel(const Args<StepArg> a, const StepFactors f)
{
    const StepArg t = a.t[tensor_of(a, (int)blockIdx.x)];
    const int64_t at = (int64_t)((int)blockIdx.x - t.first) * kChunk;
    const int n = (int)min((int64_t)kChunk, t.n - at);
    float* m = (float*)t.m + at;
    float* v = (float*)t.v + at;
    const int n4 = t.vec ? n & ~3 : 0;
    const float gf = f.grad_factor ? *f.grad_factor : 1.0f;
    constexpr int kAhead = 2;   // groups of four in flight: more take registers and gain nothing
    for (int i0 = threadIdx.x * 4; i0 < n4; i0 += kThreads * 4 * kAhead) {
        u32x4 pr[kAhead], gr[kAhead];
        f32x4 mi[kAhead], vi[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * kThreads * 4;
            if (i < n4) {
                gr[u] = load4(t.grad, t.gt, at + i);
                pr[u] = load4(t.param, t.pt, at + i);
                mi[u] = *(const f32x4*)(m + i);
                vi[u] = *(const f32x4*)(v + i);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * kThreads * 4;
            if (i < n4) {
                float p[4], g[4];
                as_float(gr[u], t.gt, g);
                as_float(pr[u], t.pt, p);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float mk = mi[u][k], vk = vi[u][k];
                    p[k] = adamw<false>(f, p[k], g[k] * gf, mk, vk);
                    mi[u][k] = mk;
                    vi[u][k] = vk;
                }
                *(f32x4*)(m + i) = mi[u];
                *(f32x4*)(v + i) = vi[u];
                store4(t.param, t.pt, at + i, p);
            }
        }
    }
    for (int i = n4 + threadIdx.x; i < n; i += kThreads) {
        float mi = m[i], vi = v[i];
        const float p = adamw<false>(f, load_as(t.param, t.pt, at + i), load_as(t.grad, t.gt, at + i) * gf, mi, vi);
        m[i] = mi;
        v[i] = vi;
        store_as(t.param, t.pt, at + i, p);
    }
}

// Maximum over the wave's lanes (row shifts and broadcasts of the vector unit), the same in all.
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    auto with = [&](uint32_t y) { x = max(x, y); };
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// A wave takes a block of 256 elements, four neighbours to a lane: the block's moments
// are decoded, stepped and scaled again without leaving the registers.  Codes come from
// the hardware's reciprocal and root, and from exact arithmetic where those leave the
// rounding open.
template <bool kFast>
__global__ __launch_bounds__(kThreads) void adamw8_kernel(const Args<Step8Arg> a, const StepFactors f)
{
    const Step8Arg t = a.t[tensor_of(a, (int)blockIdx.x)];
    const int64_t at = (int64_t)((int)blockIdx.x - t.first) * kChunk;
    const int lane = threadIdx.x & 63, i = lane * 4;
    const int blocks = (int)min((int64_t)(kChunk / kBlk), (t.n - at + kBlk - 1) / kBlk);
    const float gf = f.grad_factor ? *f.grad_factor : 1.0f;
    for (int b = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); b < blocks; b += kThreads / 64) {
        const int64_t i0 = at + (int64_t)b * kBlk;
        const int n = (int)min((int64_t)kBlk, t.n - i0);
        const bool four = t.vec && i + 4 <= n;
        int8_t* cm = (int8_t*)t.m + i0;
        uint8_t* cv = (uint8_t*)t.v + i0;
        float* ms = t.ms + i0 / kBlk;
        float* vs = t.vs + i0 / kBlk;
        float p[4] = {}, g[4] = {};
        Four<int8_t> qm = {};
        Four<uint8_t> qv = {};
        float um, uv;
        if (four) {
            const u32x4 gr = load4(t.grad, t.gt, i0 + i), pr = load4(t.param, t.pt, i0 + i);
            qm = __builtin_bit_cast(Four<int8_t>, *(const uint32_t*)(cm + i));
            qv = __builtin_bit_cast(Four<uint8_t>, *(const uint32_t*)(cv + i));
            um = *ms;
            uv = *vs;
            as_float(gr, t.gt, g);
            as_float(pr, t.pt, p);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < n) {
                    g[k] = load_as(t.grad, t.gt, i0 + i + k);
                    p[k] = load_as(t.param, t.pt, i0 + i + k);
                    qm.v[k] = cm[i + k];
                    qv.v[k] = cv[i + k];
                }
            um = *ms;
            uv = *vs;
        }
        um = m_unit(um);
        uv = v_unit(uv);
        float m[4], v[4];
        // Largest magnitudes by their bits: a NaN is larger than any number.  (Past the end all
        // is zero, and m and v stay so, unless the scale is no number.)
        uint32_t mm = 0, vm = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = m_value(qm.v[k], um);
            v[k] = v_value(qv.v[k], uv);
            p[k] = adamw<kFast>(f, p[k], g[k] * gf, m[k], v[k]);
            mm = max(mm, __float_as_uint(fabsf(m[k])));
            vm = max(vm, __float_as_uint(fabsf(v[k])));
        }
        float nms = __uint_as_float(wave_max(mm)), nvs = __uint_as_float(wave_max(vm));
        if (nms < kTiny) nms = 0.0f;
        if (nvs < kTiny) nvs = 0.0f;
        const float im = nms > 0.0f ? 1.0f / nms : 0.0f, iv = nvs > 0.0f ? 1.0f / nvs : 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            qm.v[k] = (int8_t)m_code(m[k], im);
            qv.v[k] = (uint8_t)v_code(v[k], iv);
        }
        if (four) {
            store4(t.param, t.pt, i0 + i, p);
            *(uint32_t*)(cm + i) = __builtin_bit_cast(uint32_t, qm);
            *(uint32_t*)(cv + i) = __builtin_bit_cast(uint32_t, qv);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < n) {
                    store_as(t.param, t.pt, i0 + i + k, p[k]);
                    cm[i + k] = qm.v[k];
                    cv[i + k] = qv.v[k];
                }
        }
        if (lane == 0) {
            *ms = nms;
            *vs = nvs;
        }
    }
}

// What 8-bit moments stand for: param and grad hold the fp32 outputs.
__global__ __launch_bounds__(kThreads) void moments_kernel(const Args<Step8Arg> a)
{
    const auto& t = a.t[tensor_of(a, (int)blockIdx.x)];
    const int64_t at = (int64_t)((int)blockIdx.x - t.first) * kChunk;
    const int n = (int)min((int64_t)kChunk, t.n - at);
    const int8_t* cm = (const int8_t*)t.m + at;
    const uint8_t* cv = (const uint8_t*)t.v + at;
    float* om = (float*)t.param + at;
    float* ov = (float*)t.grad + at;
    const float* ms = t.ms + at / kBlk;
    const float* vs = t.vs + at / kBlk;
    const int n4 = t.vec ? n & ~3 : 0;
    for (int i = threadIdx.x * 4; i < n4; i += kThreads * 4) {
        const Four<int8_t> qm = __builtin_bit_cast(Four<int8_t>, *(const uint32_t*)(cm + i));
        const Four<uint8_t> qv = __builtin_bit_cast(Four<uint8_t>, *(const uint32_t*)(cv + i));
        const float um = m_unit(ms[i / kBlk]), uv = v_unit(vs[i / kBlk]);
        f32x4 m, v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = m_value(qm.v[k], um);
            v[k] = v_value(qv.v[k], uv);
        }
        *(f32x4*)(om + i) = m;
        *(f32x4*)(ov + i) = v;
    }
    for (int i = n4 + threadIdx.x; i < n; i += kThreads) {
        om[i] = m_value(cm[i], m_unit(ms[i / kBlk]));
        ov[i] = v_value(cv[i], v_unit(vs[i / kBlk]));
    }
}

// Sum of the values of a workgroup of NW waves, in a fixed order.
template <int NW>
__device__ __forceinline__ double block_sum(double x, double* lds)
{
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < NW; ++w) x += lds[w];
    return x;
}

// Sums of squares in 64 bits: one of each workgroup, which the next kernel adds in their
// order, so the norm repeats to the bit.  100 MB of bf16 gradients in 300 tensors: two
// launches of 20 us, 2.6 TB/s; 7 vector instructions for 64 gradients, two of them of 64
// bits.
__global__ __launch_bounds__(kThreads) void norm_part_kernel(const Args<GradArg> a, int64_t chunk, double* __restrict__ part)
{
    __shared__ double lds[kThreads / 64];
    const GradArg t = a.t[tensor_of(a, (int)blockIdx.x)];
    const int64_t at = (int64_t)((int)blockIdx.x - t.first) * chunk;
    // 16 bytes to a load, four of them under way
    const int per = t.gt == PICTURA_F32 ? 4 : 8;
    const int64_t n = min(chunk, t.n - at), nv = t.vec ? n / per : 0;
    const u32x4* g4 = (const u32x4*)((const char*)t.grad + at * (16 / per));
    double s = 0.0;
    auto add = [&](const float* g) {
#pragma unroll
        for (int k = 0; k < 4; ++k) s = fma((double)g[k], (double)g[k], s);
    };
    for (int64_t i0 = threadIdx.x; i0 < nv; i0 += kThreads * 4) {
        u32x4 r[4] = {};
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i0 + u * kThreads < nv) r[u] = g4[i0 + u * kThreads];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float g[4];
            as_float(r[u], t.gt, g);
            add(g);
            if (per == 8) {
                as_float(u32x4{r[u][2], r[u][3], 0u, 0u}, t.gt, g);
                add(g);
            }
        }
    }
    for (int64_t i = nv * per + threadIdx.x; i < n; i += kThreads) {
        const double g = (double)load_as(t.grad, t.gt, at + i);
        s = fma(g, g, s);
    }
    s = block_sum<kThreads / 64>(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

constexpr int kNormThreads = 1024;

__global__ __launch_bounds__(kNormThreads) void norm_kernel(const double* __restrict__ part, int64_t n, float max_norm,
                                                            float* __restrict__ out)
{
    __shared__ double lds[kNormThreads / 64];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kNormThreads) s += part[i];
    s = block_sum<kNormThreads / 64>(s, lds);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(s);
        const float c = max_norm / (norm + 1e-6f);
        out[0] = norm;
        out[1] = c > 1.0f ? 1.0f : c;
    }
}

namespace {

int64_t chunks_of(int64_t n, int64_t chunk) { return (n + chunk - 1) / chunk; }

size_t size_of(int type) { return type == PICTURA_F32 ? 4 : 2; }

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool dtype_ok(int32_t t) { return t == PICTURA_F32 || t == PICTURA_BF16 || t == PICTURA_F16; }

// Split the tensors over launches of as many tensors as their arguments hold and 2^22
// workgroups of `chunk` elements; a tensor beyond that is taken in parts.
// launch(args, blocks).
template <class Arg, class Fill, class Launch>
void for_launches(const pictura_adamw_tensor* ts, int32_t count, int64_t chunk, Fill fill, Launch launch)
{
    constexpr int64_t kMostBlocks = 1 << 22;
    Args<Arg> a;
    a.count = 0;
    int64_t blocks = 0;
    auto flush = [&] {
        if (a.count) launch(a, (unsigned)blocks);
        a.count = 0;
        blocks = 0;
    };
    for (int32_t k = 0; k < count; ++k) {
        int64_t at = 0;
        while (at < ts[k].n) {
            const int64_t left = chunks_of(ts[k].n - at, chunk), room = kMostBlocks - blocks;
            const int64_t take = left < room ? left : room;
            Arg& t = a.t[a.count];
            t.n = ts[k].n - at < take * chunk ? ts[k].n - at : take * chunk;
            t.first = (int32_t)blocks;
            fill(t, k, at);
            ++a.count;
            blocks += take;
            at += take * chunk;
            if (a.count == Args<Arg>::kMost || blocks == kMostBlocks) flush();
        }
    }
    flush();
}

void fill_step(StepArg& t, const pictura_adamw_tensor& s, int64_t at, int bits)
{
    t.param = (char*)s.param + at * size_of(s.param_dtype);
    t.grad = (const char*)s.grad + at * size_of(s.grad_dtype);
    const size_t b = bits == 8 ? 1 : 4;
    t.m = (char*)s.exp_avg + at * b;
    t.v = (char*)s.exp_avg_sq + at * b;
    t.pt = (uint8_t)s.param_dtype;
    t.gt = (uint8_t)s.grad_dtype;
    t.vec = aligned(t.param, 4 * size_of(s.param_dtype)) && aligned(t.grad, 4 * size_of(s.grad_dtype)) &&
            aligned(t.m, 4 * b) && aligned(t.v, 4 * b);
}

void fill_scales(Step8Arg& t, const pictura_adamw_tensor& s, int64_t at)
{
    t.ms = s.exp_avg_scale + at / kBlk;
    t.vs = s.exp_avg_sq_scale + at / kBlk;
}

// Elements of a workgroup of the norm: at most some 2,048 workgroups (eight to a CU),
// whose sums one more adds up.  Four times as many, with a quarter of the elements each,
// take 21 us where these take 20 (above).
int64_t norm_chunk(const pictura_adamw_tensor* ts, int32_t count)
{
    int64_t n = 0;
    for (int32_t k = 0; k < count; ++k) n += ts[k].n;
    const int64_t c = chunks_of(n, 2048);
    return c < kChunk ? kChunk : chunks_of(c, kChunk) * kChunk;
}

constexpr int64_t kMostElements = 1ll << 48;

bool moments_ok(const pictura_adamw_tensor& t, int bits)
{
    if (!t.exp_avg || !t.exp_avg_sq) return false;
    if (bits == 32) return aligned(t.exp_avg, 4) && aligned(t.exp_avg_sq, 4);
    return t.exp_avg_scale && t.exp_avg_sq_scale && aligned(t.exp_avg_scale, 4) && aligned(t.exp_avg_sq_scale, 4);
}

bool grads_ok(const pictura_adamw_tensor* ts, int32_t count)
{
    if (count < 0 || (count > 0 && !ts)) return false;
    for (int32_t k = 0; k < count; ++k) {
        const pictura_adamw_tensor& t = ts[k];
        if (t.n < 0 || t.n > kMostElements || !dtype_ok(t.grad_dtype)) return false;
        if (t.n > 0 && (!t.grad || !aligned(t.grad, size_of(t.grad_dtype)))) return false;
    }
    return true;
}

pictura_status launched() { return hipGetLastError() == hipSuccess ? PICTURA_OK : PICTURA_EDEVICE; }

}  // namespace
}  // namespace pictura

using namespace pictura;

extern "C" {

pictura_status pictura_grad_norm_workspace(const pictura_adamw_tensor* tensors, int32_t count, uint64_t* bytes)
{
    if (!bytes || count < 0 || (count > 0 && !tensors)) return PICTURA_EINVAL;
    for (int32_t k = 0; k < count; ++k)
        if (tensors[k].n < 0 || tensors[k].n > kMostElements) return PICTURA_EINVAL;
    const int64_t chunk = norm_chunk(tensors, count);
    int64_t n = 0;
    for (int32_t k = 0; k < count; ++k) n += chunks_of(tensors[k].n, chunk);
    *bytes = (uint64_t)(n > 0 ? n : 1) * sizeof(double);
    return PICTURA_OK;
}

pictura_status pictura_grad_norm(const pictura_adamw_tensor* tensors, int32_t count, float max_norm, void* workspace,
                                 uint64_t workspace_bytes, float* out, void* stream)
{
    if (!grads_ok(tensors, count) || !out || !workspace || !aligned(out, 4) || !aligned(workspace, 256)) return PICTURA_EINVAL;
    if (!(max_norm >= 0.0f)) return PICTURA_EINVAL;
    uint64_t need = 0;
    pictura_status st = pictura_grad_norm_workspace(tensors, count, &need);
    if (st != PICTURA_OK) return st;
    if (workspace_bytes < need) return PICTURA_EINVAL;
    hipStream_t s = (hipStream_t)stream;
    double* part = (double*)workspace;
    int64_t n = 0;
    const int64_t chunk = norm_chunk(tensors, count);
    for_launches<GradArg>(
        tensors, count, chunk,
        [&](GradArg& t, int32_t k, int64_t at) {
            t.grad = (const char*)tensors[k].grad + at * size_of(tensors[k].grad_dtype);
            t.gt = (uint8_t)tensors[k].grad_dtype;
            t.vec = aligned(t.grad, 16);
        },
        [&](const Args<GradArg>& a, unsigned blocks) {
            hipLaunchKernelGGL(norm_part_kernel, dim3(blocks), dim3(kThreads), 0, s, a, chunk, part + n);
            n += blocks;
        });
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kNormThreads), 0, s, part, n, max_norm, out);
    return launched();
}

pictura_status pictura_adamw_step(const pictura_adamw* how, const pictura_adamw_tensor* tensors, int32_t count,
                                  void* stream)
{
    if (!how || !grads_ok(tensors, count)) return PICTURA_EINVAL;
    if (how->bits != 32 && how->bits != 8) return PICTURA_EINVAL;
    if (!(how->beta1 >= 0.0 && how->beta1 < 1.0 && how->beta2 >= 0.0 && how->beta2 < 1.0) || how->step < 1) return PICTURA_EINVAL;
    if (!std::isfinite(how->lr) || !(how->eps >= 0.0) || !std::isfinite(how->weight_decay)) return PICTURA_EINVAL;
    for (int32_t k = 0; k < count; ++k) {
        const pictura_adamw_tensor& t = tensors[k];
        if (!dtype_ok(t.param_dtype)) return PICTURA_EINVAL;
        if (t.n > 0 && (!t.param || !aligned(t.param, size_of(t.param_dtype)) || !moments_ok(t, how->bits)))
            return PICTURA_EINVAL;
    }
    hipStream_t s = (hipStream_t)stream;
    const double bc1 = 1.0 - std::pow(how->beta1, (double)how->step), bc2 = 1.0 - std::pow(how->beta2, (double)how->step);
    const StepFactors f{(float)how->beta1, (float)(1.0 - how->beta1), (float)how->beta2, (float)(1.0 - how->beta2),
                        (float)(1.0 / std::sqrt(bc2)), (float)how->eps, (float)(1.0 - how->lr * how->weight_decay),
                        (float)(how->lr / bc1), how->grad_factor};
    if (how->bits == 32)
        for_launches<StepArg>(
            tensors, count, kChunk, [&](StepArg& t, int32_t k, int64_t at) { fill_step(t, tensors[k], at, 32); },
            [&](const Args<StepArg>& a, unsigned blocks) {
                hipLaunchKernelGGL(adamw32_kernel, dim3(blocks), dim3(kThreads), 0, s, a, f);
            });
    else {
        const auto kernel = f.eps >= kLeastEps ? adamw8_kernel<true> : adamw8_kernel<false>;
        for_launches<Step8Arg>(
            tensors, count, kChunk,
            [&](Step8Arg& t, int32_t k, int64_t at) {
                fill_step(t, tensors[k], at, 8);
                fill_scales(t, tensors[k], at);
            },
            [&](const Args<Step8Arg>& a, unsigned blocks) {
                hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, s, a, f);
            });
    }
    return launched();
}

pictura_status pictura_adamw_moments(const pictura_adamw_tensor* tensors, int32_t count, float* const* exp_avg_out,
                                     float* const* exp_avg_sq_out, void* stream)
{
    if (count < 0 || (count > 0 && (!tensors || !exp_avg_out || !exp_avg_sq_out))) return PICTURA_EINVAL;
    for (int32_t k = 0; k < count; ++k) {
        const pictura_adamw_tensor& t = tensors[k];
        if (t.n < 0 || t.n > kMostElements) return PICTURA_EINVAL;
        if (t.n > 0 && (!moments_ok(t, 8) || !exp_avg_out[k] || !exp_avg_sq_out[k] || !aligned(exp_avg_out[k], 4) ||
                        !aligned(exp_avg_sq_out[k], 4)))
            return PICTURA_EINVAL;
    }
    hipStream_t s = (hipStream_t)stream;
    for_launches<Step8Arg>(
        tensors, count, kChunk,
        [&](Step8Arg& t, int32_t k, int64_t at) {
            t.param = exp_avg_out[k] + at;
            t.grad = exp_avg_sq_out[k] + at;
            t.m = (char*)tensors[k].exp_avg + at;
            t.v = (char*)tensors[k].exp_avg_sq + at;
            t.vec = aligned(t.param, 16) && aligned(t.grad, 16) && aligned(t.m, 4) && aligned(t.v, 4);
            fill_scales(t, tensors[k], at);
        },
        [&](const Args<Step8Arg>& a, unsigned blocks) {
            hipLaunchKernelGGL(moments_kernel, dim3(blocks), dim3(kThreads), 0, s, a);
        });
    return launched();
}

}  // extern "C"
