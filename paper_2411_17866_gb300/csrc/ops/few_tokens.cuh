// The loss of a language-model head and its gradient for a few tokens (scoring or training on single tokens): W is read
// row by row as it lies, whatever its type and alignment, and multiplied in f32 on the ordinary cores.  Nothing is
// gathered, packed or padded; the time is that of reading W (once for the loss, twice for the gradient) and writing dW.
//
// Logits: a warp takes R rows of W at a time, a thread 16 bytes of each, against the rows of h in shared memory; R x TN
// sums per thread are then added over the warp by halves, after which a thread holds one or two logits, always of the
// same token.  Per loaded piece of h there are R multiply-adds a value: below R = 4 reading h would take longer than W.
#pragma once

#include "ops_host.h"

namespace dsm {
namespace ops {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The power of two that the exponentials of logits up to `top` are divided by: a whole number, so that the division and
// later changes of it are exact.
__device__ __forceinline__ float reference(float top) { return top == -INFINITY ? 0.f : rintf(top * kLog2e); }

// What takes a sum over logits up to `top` to the reference `ref` of a larger one.  0 for a sum of nothing (top = -infinity),
// however far below zero the logits lie: its own reference of 0 would make 2^-ref of it, infinite below logits of -88.
__device__ __forceinline__ float rescale(float top, float ref) { return exp2_fast(rintf(top * kLog2e) - ref); }

// (largest logit, sum of 2^(s log2(e) - reference)) of two parts.
__device__ __forceinline__ float2 joined(float2 a, float2 b) {
    const float top = fmaxf(a.x, b.x), ref = reference(top);
    return make_float2(top, fmaf(a.y, rescale(a.x, ref), b.y * rescale(b.x, ref)));
}
__device__ __forceinline__ float log_sum(float2 v) { return v.x + kLn2 * (log2f(v.y) + fmaf(-kLog2e, v.x, reference(v.x))); }

struct FewArgs {
    const void *h, *w, *targets;
    uint64_t h_stride, w_stride;
    int64_t ignore;
    uint32_t tokens, vocab, width;
    int target64, vec;           // vec: rows of W start on 16-byte boundaries
    uint32_t* status;
    // loss
    float2* partial;             // [CTAs][TN]
    float* target_logit;         // [TN]
    float *loss, *lse;
    // gradient
    const float *lse_in, *grad_loss;
    uint64_t grad_stride;
    float* g;                    // [vocab][TN]: G
    float* sum;                  // [splits][TN][ld]: parts of dh
    void *dh, *dw;
    uint64_t dh_stride, dw_stride;
    uint32_t ld, splits;
    int out_vec;                 // rows of dW as vec
};

__device__ __forceinline__ int64_t few_target(const FewArgs& p, uint32_t t) {
    return p.target64 ? static_cast<const int64_t*>(p.targets)[t] : static_cast<const int32_t*>(p.targets)[t];
}

constexpr int kOuterThreads = 128;
// Columns of a thread in k_ce_few_outer: 16 bytes where the registers allow it.
template <typename T>
__host__ __device__ constexpr int few_columns(int tn) {
    return tn <= 4 ? 16 / sizeof(T) : tn <= 8 ? 4 : 2;
}

// Threads of a CTA, by the sums that each holds: of 128 registers a thread 64 sums spill.
__host__ __device__ constexpr int few_threads(int sums) { return sums > 32 ? 384 : 512; }

// Places of a row of h in shared memory: a thread reads 4 values at a time next to its neighbours' (16-bit W: the second
// halves of groups of 8 in a plane of their own).
template <typename T>
__host__ __device__ constexpr uint32_t few_group() {
    return 16 / sizeof(T);
}
template <typename T>
__host__ __device__ inline uint32_t few_padded(uint32_t width) {
    return (width + few_group<T>() * 32 - 1) / (few_group<T>() * 32) * (few_group<T>() * 32);
}
template <typename T>
__device__ __forceinline__ uint32_t few_place(uint32_t k, uint32_t padded) {
    constexpr uint32_t kG = few_group<T>();
    return kG == 4 ? k : (k % 8 / 4) * (padded / 2) + k / 8 * 4 + k % 4;
}

// Value i of a piece of W, held as 32-bit words.
template <typename T>
__device__ __forceinline__ float few_value(const uint32_t* words, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(words[i]);
    return __uint_as_float(i % 2 ? words[i / 2] & 0xffff0000u : words[i / 2] << 16);
}

template <int N>
__device__ __forceinline__ void add_over_warp(float (&v)[N], uint32_t lane, uint32_t& first, int& left) {
    // v[0..N) over 32 lanes by halves: a lane keeps the upper half of what it has if its bit is set
    first = 0;
    left = N;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        if (left > 1) {
            left /= 2;
            const bool upper = lane & o;
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                if (i < left) {
                    const float send = upper ? v[i] : v[i + left], keep = upper ? v[i + left] : v[i];
                    v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
            first += upper ? left : 0;
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        }
    }
}

// The logits of up to TN tokens against all rows of W: their partial results for the loss, or G.
template <typename T, int TN, int R, bool GRAD>
__global__ void __launch_bounds__(few_threads(R * TN), 1) k_ce_few(const __grid_constant__ FewArgs p) {
    constexpr int kFewThreads = few_threads(R * TN);
    extern __shared__ __align__(16) float hs[];
    __shared__ float2 parts[kFewThreads / 32][32][2];
    constexpr uint32_t kG = few_group<T>();
    constexpr int N = R * TN, kHeld = N > 32 ? N / 32 : 1;
    static_assert(N <= 64 && (N & (N - 1)) == 0, "sums per thread");
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, padded = few_padded<T>(p.width);
    wait_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;
    // rows of h that take no part are zero, whatever they hold
    for (uint32_t t = 0; t < TN; ++t) {
        const bool kept = t < p.tokens && few_target(p, t) != p.ignore;
        const T* row = static_cast<const T*>(p.h) + t * p.h_stride;
        for (uint32_t k = threadIdx.x; k < padded; k += kFewThreads)
            hs[t * padded + few_place<T>(k, padded)] = kept && k < p.width ? to_float(row[k]) : 0.f;
    }
    __syncthreads();

    // which of the R x TN sums this thread ends up with
    uint32_t first;
    {
        float none[N] = {};
        int left;
        add_over_warp(none, lane, first, left);
    }
    // (N < 32: several threads hold the same one)
    constexpr uint32_t kSame = N >= 32 ? 1 : 32 / N;
    const bool mine = lane % kSame == 0;
    float2 run[kHeld];
    int64_t y[kHeld];
    float a[kHeld], ref[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const uint32_t t = (first + i) % TN;
        run[i] = make_float2(-INFINITY, 0.f);
        y[i] = t < p.tokens ? few_target(p, t) : p.ignore;
        a[i] = ref[i] = 0.f;
        if (GRAD && t < p.tokens && y[i] != p.ignore) {
            a[i] = p.grad_loss[t * p.grad_stride];
            ref[i] = p.lse_in[t];
        }
    }

    const T* w = static_cast<const T*>(p.w);
    const uint32_t step = gridDim.x * (kFewThreads / 32) * R;
    uint32_t v0 = (blockIdx.x * (kFewThreads / 32) + warp) * R;
    // the next piece of every row is under way while this one is multiplied, over the ends of rows as well
    uint4 next[R];
    auto load = [&](uint32_t v, uint32_t k) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const T* at = w + uint64_t(v + r < p.vocab ? v + r : p.vocab - 1) * p.w_stride + k;
            if (k + kG <= p.width) {
                next[r] = __ldg(reinterpret_cast<const uint4*>(at));
            } else {
                __align__(16) T part[kG] = {};
                for (uint32_t i = 0; k + i < p.width; ++i) part[i] = at[i];
                next[r] = *reinterpret_cast<uint4*>(part);
            }
        }
    };
    if (p.vec && v0 < p.vocab) load(v0, lane * kG);
    for (; v0 < p.vocab; v0 += step) {
        float sum[N];
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.f;
        if (p.vec) {
            for (uint32_t k0 = 0; k0 < p.width; k0 += 32 * kG) {
                uint4 raw[R];
#pragma unroll
                for (int r = 0; r < R; ++r) raw[r] = next[r];
                const bool more = k0 + 32 * kG < p.width;
                if (more || v0 + step < p.vocab) load(more ? v0 : v0 + step, (more ? k0 + 32 * kG : 0) + lane * kG);
                const uint32_t k = k0 + lane * kG;   // (h is zero where it lies beyond the last)
#pragma unroll
                for (uint32_t q = 0; q < kG / 4; ++q)
#pragma unroll
                    for (int t = 0; t < TN; ++t) {
                        const float4 x = *reinterpret_cast<const float4*>(hs + t * padded + q * (padded / 2) + k / kG * 4);
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const uint32_t* word = reinterpret_cast<const uint32_t*>(&raw[r]);
                            float& s = sum[r * TN + t];
                            s = fmaf(few_value<T>(word, 4 * q), x.x, s);
                            s = fmaf(few_value<T>(word, 4 * q + 1), x.y, s);
                            s = fmaf(few_value<T>(word, 4 * q + 2), x.z, s);
                            s = fmaf(few_value<T>(word, 4 * q + 3), x.w, s);
                        }
                    }
            }
        } else {
#pragma unroll 4
            for (uint32_t k = lane; k < p.width; k += 32) {
                float e[R];
#pragma unroll
                for (int r = 0; r < R; ++r) e[r] = to_float(w[uint64_t(v0 + r < p.vocab ? v0 + r : v0) * p.w_stride + k]);
#pragma unroll
                for (int t = 0; t < TN; ++t) {
                    const float x = hs[t * padded + few_place<T>(k, padded)];
#pragma unroll
                    for (int r = 0; r < R; ++r) sum[r * TN + t] = fmaf(e[r], x, sum[r * TN + t]);
                }
            }
        }
        uint32_t at;
        int left;
        add_over_warp(sum, lane, at, left);
        if (!mine) continue;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const uint32_t v = v0 + (first + i) / TN, t = (first + i) % TN;
            if (v >= p.vocab) continue;
            if constexpr (GRAD) {
                float g = exp2_fast((sum[i] - ref[i]) * kLog2e);
                if (v == y[i]) g -= 1.f;
                p.g[uint64_t(v) * TN + t] = t < p.tokens && y[i] != p.ignore ? g * a[i] : 0.f;
            } else {
                run[i] = joined(run[i], make_float2(sum[i], exp2_fast(fmaf(sum[i], kLog2e, -reference(sum[i])))));
                if (v == y[i]) p.target_logit[t] = sum[i];
            }
        }
    }
    if constexpr (!GRAD) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) parts[warp][lane][i] = mine ? run[i] : make_float2(-INFINITY, 0.f);
        // a thread's token: (first + i) % TN, first from the bits of its lane
        __shared__ uint8_t token_of[32][2];
        if (warp == 0)
#pragma unroll
            for (int i = 0; i < kHeld; ++i) token_of[lane][i] = static_cast<uint8_t>((first + i) % TN);
        __syncthreads();
        // a warp to a token
        for (uint32_t t = warp; t < TN; t += kFewThreads / 32) {
            float2 v = make_float2(-INFINITY, 0.f);
            for (int i = 0; i < kHeld; ++i)
                if (token_of[lane][i] == t)
                    for (int k = 0; k < kFewThreads / 32; ++k) v = joined(v, parts[k][lane][i]);
            for (int o = 16; o; o >>= 1)
                v = joined(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
            if (lane == 0) p.partial[blockIdx.x * TN + t] = v;
        }
    }
}

// The loss from the CTAs' partial results, a warp to a token.
template <int TN>
__global__ void __launch_bounds__(32 * TN) k_ce_few_join(const __grid_constant__ FewArgs p, uint32_t ctas) {
    wait_previous();
    const uint32_t t = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (t >= p.tokens) return;
    float2 v = make_float2(-INFINITY, 0.f);
    for (uint32_t i = lane; i < ctas; i += 32) v = joined(v, p.partial[i * TN + t]);
    for (int o = 16; o; o >>= 1)
        v = joined(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
    if (lane) return;
    const int64_t y = few_target(p, t);
    const bool kept = y != p.ignore, known = y >= 0 && y < p.vocab;
    const float lse = log_sum(v);
    p.lse[t] = !kept ? 0.f : known ? lse : NAN;
    p.loss[t] = !kept ? 0.f : known ? lse - p.target_logit[t] : NAN;
}

// dW = G^T h and parts of dh = G W.  A thread has C columns, of h and of the sums in registers, and walks down its CTA's
// part of the rows of W, kRows at a time with the next ones' loads under way; G comes by shared memory, 64 rows at a time.
// VEC: the columns are neighbours, one load of all.  Else (rows of W or dW that do not start on 16-byte boundaries) they are
// kOuterThreads apart and neighbouring threads have neighbouring ones.
template <typename T, int TN, int C, bool VEC>
__global__ void __launch_bounds__(kOuterThreads) k_ce_few_outer(const __grid_constant__ FewArgs p) {
    __shared__ __align__(16) float gs[2][64 * TN];
    constexpr int kMine = 64 * TN / kOuterThreads > 1 ? 64 * TN / kOuterThreads : 1;
    wait_previous();
    const uint32_t c = blockIdx.x * (kOuterThreads * C) + threadIdx.x * (VEC ? C : 1);
    constexpr uint32_t kApart = VEC ? 1 : kOuterThreads;
    const uint32_t v0 = static_cast<uint32_t>(uint64_t(p.vocab) * blockIdx.y / p.splits);
    const uint32_t v1 = static_cast<uint32_t>(uint64_t(p.vocab) * (blockIdx.y + 1) / p.splits);
    float h[TN][C], sum[TN][C];
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        const bool kept = t < p.tokens && few_target(p, t) != p.ignore;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            h[t][i] = kept && c + i * kApart < p.width ? to_float(static_cast<const T*>(p.h)[t * p.h_stride + c + i * kApart]) : 0.f;
            sum[t][i] = 0.f;
        }
    }
    const bool any = c < p.width, whole = VEC && c + C <= p.width;
    const T* w = static_cast<const T*>(p.w) + (any ? c : 0);
    T* dw = static_cast<T*>(p.dw) + c;
    // C values as 32-bit words (not VEC: a word each): as an array of 16-bit values their copies would wait for the loads
    constexpr int kRows = 8, kWords = VEC ? C * sizeof(T) / 4 : C;
    struct alignas(kWords * 4) Words {
        uint32_t v[kWords];
    };
    Words next[kRows];
    auto load = [&](uint32_t v) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const T* at = w + uint64_t(v + r < v1 ? v + r : v1 - 1) * p.w_stride;
            if constexpr (!VEC) {
#pragma unroll
                for (int i = 0; i < C; ++i) {   // (predicated: a branch around whole sets of columns took 129 us for 71)
                    next[r].v[i] = 0;
                    if constexpr (sizeof(T) == 4) {
                        if (c + i * kApart < p.width) next[r].v[i] = __float_as_uint(at[i * kApart]);
                    } else {
                        if (c + i * kApart < p.width) next[r].v[i] = reinterpret_cast<const uint16_t*>(at)[i * kApart];
                    }
                }
            } else if (whole) {
                next[r] = *reinterpret_cast<const Words*>(at);
            } else {
                __align__(16) T part[C];
#pragma unroll
                for (int i = 0; i < C; ++i) part[i] = c + i < p.width ? at[i] : round_to<T>(0.f);
                next[r] = *reinterpret_cast<const Words*>(part);
            }
        }
    };
    // G of the 64 rows from v on: into registers, and later into its half of gs
    float mine[kMine];
    auto fetch = [&](uint32_t v) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const uint32_t at = threadIdx.x + i * kOuterThreads;
            mine[i] = at < 64 * TN && v + at / TN < v1 ? p.g[uint64_t(v) * TN + at] : 0.f;
        }
    };
    fetch(v0);
    load(v0);
    for (uint32_t v = v0; v < v1; v += kRows) {
        const uint32_t half = (v - v0) / 64 & 1;
        if ((v - v0) % 64 == 0) {
#pragma unroll
            for (int i = 0; i < kMine; ++i)
                if (threadIdx.x + i * kOuterThreads < 64 * TN) gs[half][threadIdx.x + i * kOuterThreads] = mine[i];
            __syncthreads();   // (the other half was last read before the barrier ahead of this one's)
            fetch(v + 64);
        }
        Words e[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) e[r] = next[r];
        if (v + kRows < v1) load(v + kRows);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (!any || v + r >= v1) break;
            const float* g = gs[half] + ((v - v0) % 64 + r) * TN;
            float x[C] = {}, in[C];
#pragma unroll
            for (int i = 0; i < C; ++i)
                in[i] = VEC ? few_value<T>(e[r].v, i) : __uint_as_float(sizeof(T) == 4 ? e[r].v[i] : e[r].v[i] << 16);
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                const float gt = g[t];
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    sum[t][i] = fmaf(gt, in[i], sum[t][i]);
                    x[i] = fmaf(gt, h[t][i], x[i]);
                }
            }
            if (!p.dw) continue;
            T* to = dw + uint64_t(v + r) * p.dw_stride;
            __align__(16) T out[C];
#pragma unroll
            for (int i = 0; i < C; ++i) out[i] = round_to<T>(x[i]);
            if (whole) {
                *reinterpret_cast<Words*>(to) = *reinterpret_cast<Words*>(out);
            } else {
#pragma unroll
                for (int i = 0; i < C; ++i)
                    if (c + i * kApart < p.width) to[i * kApart] = out[i];
            }
        }
    }
    if (!p.dh) return;
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (c + i * kApart < p.width) p.sum[(uint64_t(blockIdx.y) * TN + t) * p.ld + c + i * kApart] = sum[t][i];
}

// dh from its parts: 32 columns of a token by 32 warps, each with every 32nd part, in a fixed order.
template <typename T, int TN>
__global__ void __launch_bounds__(1024) k_ce_few_sum(const __grid_constant__ FewArgs p) {
    __shared__ float parts[32][33];
    wait_previous();
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, t = blockIdx.y, c = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (c < p.width) {
#pragma unroll 8
        for (uint32_t s = warp; s < p.splits; s += 32) v += p.sum[(uint64_t(s) * TN + t) * p.ld + c];
    }
    parts[warp][lane] = v;
    __syncthreads();
    // a warp to a column: its 32 parts
    v = parts[lane][warp];
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const uint32_t column = blockIdx.x * 32 + warp;
    if (lane == 0 && column < p.width)
        static_cast<T*>(p.dh)[t * p.dh_stride + column] = few_target(p, t) != p.ignore ? round_to<T>(v) : round_to<T>(0.f);
}

}  // namespace ops
}  // namespace dsm
