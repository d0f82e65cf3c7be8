// What the policy's entries hand to the kernels of each type of logits.
#pragma once

#include "pictura.h"
#include "pictura_internal.h"

namespace pictura {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

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

struct Work {
    double* part;         // sums of loss_moments_kernel
    int32_t parts;
    double* sums;
    uint32_t* done;
};

template <class T>
void launch_sample(const Rows& R, const Sampling& S, const float* uniform, int64_t* action, float* logp, hipStream_t s);
template <class T>
void launch_loss(const Rows& R, const Batch& b, const Work& k, hipStream_t s);
int64_t loss_blocks(int64_t rows, int32_t actions);

// Lanes that hold a row of up to 64 actions.
inline int group_lanes(int32_t actions) { return actions <= 8 ? 8 : actions <= 16 ? 16 : actions <= 32 ? 32 : 64; }

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// What the entries check.
inline size_t size_of(int32_t t) { return t == PICTURA_F32 ? 4 : 2; }

inline bool logits_ok(const pictura_logits* l)
{
    if (!l || (l->dtype != PICTURA_F32 && l->dtype != PICTURA_BF16 && l->dtype != PICTURA_F16)) return false;
    if (l->actions < 1 || l->actions > PICTURA_MAX_ACTIONS || l->rows < 0 || l->rows > 0x7FFFFFFFll) return false;
    if (l->rows == 0) return true;
    if (l->stride < l->actions && l->rows > 1) return false;
    if (l->mask && l->mask_stride != 0 && l->mask_stride < l->actions && l->rows > 1) return false;
    return l->data && aligned(l->data, size_of(l->dtype));
}

inline Rows rows_of(const pictura_logits& l) { return Rows{l.data, l.stride, l.mask, l.mask_stride, l.rows, l.actions}; }

}  // namespace pictura
