// What the policy's entries hand to the kernels of each type of logits.
#pragma once

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

}  // namespace pictura
