// What the kernels of dsm_orthogonalize share: the momentum's update and the norm.
#pragma once

#include "ops_host.h"

namespace dsm {
namespace ops {
namespace {

constexpr float kScale = 4096.f;        // of X, A and B as f16
// Squares are summed of values times kUp, and apart of those above kBig times kDown: both stay below 2^43, so that 2^40
// squares (the most a matrix has) do not overflow, and down to 2^-84 a value's square is a normal number.
constexpr float kBig = 0x1p22f, kUp = 0x1p21f, kDown = 0x1p-85f;
constexpr uint32_t kUpdateBlocks = 256; // most CTAs per matrix of the update kernel, each with a partial sum

struct Strides {
    int64_t batch, row, col;
};

struct UpdateArgs {
    const void* g;
    float* momentum;
    float* u;                 // [count][rows][ld] f32, of the strided form
    float2* partial;          // [count][kUpdateBlocks]: sums of squares, see kBig
    uint32_t *status, *barrier;   // set to zero
    Strides gs, ms;
    uint32_t rows, cols, ld;
    float mu;
    int nesterov;
    int has_momentum;
};

__device__ __forceinline__ void add_square(float v, float2& sum) {
    const bool big = fabsf(v) > kBig;
    const float t = v * (big ? kDown : kUp);
    if (big) sum.y = fmaf(t, t, sum.y);
    else sum.x = fmaf(t, t, sum.x);
}

// What takes u to X_0: u * by * factor.  (Two factors: the norm of large values, and its inverse, may be outside f32's range.)
struct Unit {
    float by, factor;
    __device__ __forceinline__ float operator()(float u) const { return u * by * factor; }
};

// From the sums of u's squares.  A NaN among them stays NaN, and an infinity (which no finite values add up to) becomes one:
// its inverse would be 0 and all finite values of the matrix with it.
__device__ __forceinline__ Unit to_unit(float2 sum, float eps) {
    constexpr float kApart = kDown / kUp;
    const bool big = sum.y > 0.f;
    const float norm = big ? sqrtf(fmaf(sum.x * kApart, kApart, sum.y)) : sqrtf(sum.x) * (1.f / kUp);   // times `by`
    const float by = big ? kDown : 1.f, least = fmaxf(eps * by, 0x1p-126f);
    return Unit{by, norm == INFINITY ? NAN : 1.f / (norm < least ? least : norm)};
}

// Sums `v` over the CTA (256 threads) in a fixed order; the result is in every thread.
__device__ __forceinline__ float2 cta_sum(float2 v, float2* shared) {
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = v;
    __syncthreads();
    float2 r = make_float2(0.f, 0.f);
    for (int i = 0; i < 8; ++i) {
        r.x += shared[i].x;
        r.y += shared[i].y;
    }
    __syncthreads();
    return r;
}

// The momentum's update of one element, and u.
__device__ __forceinline__ float updated(const UpdateArgs& p, float g, float& m) {
    m = fmaf(p.mu, m, g);
    return p.nesterov ? fmaf(p.mu, m, g) : m;
}

}  // namespace
}  // namespace ops
}  // namespace dsm
