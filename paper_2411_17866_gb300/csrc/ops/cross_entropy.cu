// dsm_linear_cross_entropy, dsm_linear_cross_entropy_grad: the loss of a language-model head, h W^T against targets, and
// its gradient, over the vocabulary in pieces: no [tokens, vocabulary] array is kept from the loss to the gradient.
//
//   s_tv = h_t . W_v,  lse_t = log sum_v exp s_tv,  loss_t = lse_t - s_t,y_t
//   G_tv = a_t (exp(s_tv - lse_t) - [v = y_t]),  dh = G W,  dW = G^T h
//
// Tokens whose target is the ignored one take no part: the kept rows of h are gathered first, and every product runs
// over those alone (so that neither their number nor what lies in ignored rows matters).
//
// Loss: one product whose epilogue keeps, per row and tile of the vocabulary, the maximum and the sum of exponentials;
// the partial results are joined in a fixed order.  Gradient: per piece of the vocabulary the logits again, whose
// epilogue writes that piece of G, then the piece's contribution to dh (f32, added up over the pieces and over parts of
// the vocabulary where there are few rows) and its rows of dW.
//
// Numbers.  16-bit operands are multiplied as they are (bf16, f32 accumulators), G is rounded to bf16.  A token's G adds up
// to zero, so what W's rows have in common drops out of dh; of the rounded G a rest s_t is left, and dh takes
// G W - s_t W_y, which puts the rest on the target and with it back to zero.  (All rows of W with a common part that moves
// the logits to -120: dh was off by 6.5 %, and is by 0.3 %.)
//
// 32-bit operands are kept as pairs hi + lo of f16 (22 bits) and multiplied in three terms.  Every row of h and of W is scaled
// by a power of two of its own so that its largest value lies just below f16's range.  G is kept without grad_loss,
// p_tv - [v = y_t], and twice: for dh with the scales of W's rows, which its product sums over (grad_loss_t comes last), and
// for dW as it is, against grad_loss_t h_t under one scale for all.  So neither a row of W nor a token sets the precision of
// another's gradient: G and grad_loss_t h_t keep 22 bits down to 2^-17 of their largest value, and 2^-39 of that as an
// absolute error below.  (G once, with both scales folded in: rows of W or h that are zero, or much smaller than the others,
// cost dh and dW up to 31 bits.)  Statistics, lse and the sums for dh are in f32.
#include <type_traits>

#include "few_tokens.cuh"
#include "ops_host.h"

namespace dsm {
namespace ops {
namespace {

constexpr uint32_t kSms = 152;         // of a GB300: what work is divided for
constexpr uint32_t kRowPad = 256;      // rows of the gathered h and of G come in multiples of this
constexpr int kTopExponent = 14;       // of the largest value of a scaled row

// floor(log2 |v|), within the range in which 2^(kTopExponent - it) and its inverse are normal numbers.
constexpr int kLeastExponent = kTopExponent - 126;
__device__ __forceinline__ int exponent(float v) {
    const int e = static_cast<int>(__float_as_uint(v) >> 23 & 255) - 127;
    return e < kLeastExponent ? kLeastExponent : e > 127 ? 127 : e;
}
__device__ __forceinline__ float power(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// v 2^e for e in [-252, 254]
__device__ __forceinline__ float times_power(float v, int e) { return v * power(e / 2) * power(e - e / 2); }

// The same of grad_loss, whose inverse has to be normal.
__device__ __forceinline__ int grad_exponent(float a) { return min(exponent(a), 126); }

// What 32-bit operands are scaled by: the largest exponents of grad_loss_t times the inverse scale of h_t, and of the inverse
// scales of W.
struct Scales {
    int h, w;
};

// 16-bit operand planes of rows of h or W: bf16, or f16 pairs with the inverse of every row's scale.
struct Planes {
    uint16_t *hi, *lo;
    float* inverse;
    uint32_t ld;              // a multiple of 8
};

// One row, by one warp.  Returns the exponent of the inverse of its scale (0 for bf16); a row of zeros has the least one, so
// that it is nobody's largest.
template <typename T>
__device__ __forceinline__ int copy_row(const T* src, uint32_t width, const Planes& to, uint64_t row, uint32_t lane) {
    const uint64_t at = row * to.ld;
    constexpr bool kPair = sizeof(T) == 4;
    const bool vec = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
    auto eight = [&](uint32_t k, T (&v)[8]) {
        if (vec && k + 8 <= width) {
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
                reinterpret_cast<uint4*>(v)[i] = *(reinterpret_cast<const uint4*>(src + k) + i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < width ? src[k + i] : round_to<T>(0.f);
        }
    };
    float scale = 1.f;
    int inverse = 0;
    if constexpr (kPair) {
        float most = 0.f;
#pragma unroll 2
        for (uint32_t k = lane * 8; k < to.ld; k += 256) {
            __align__(16) T v[8];
            eight(k, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = fabsf(v[i]);
                if (x < INFINITY) most = fmaxf(most, x);   // what is not finite stays so under any scale
            }
        }
        most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
        inverse = exponent(most) - kTopExponent;   // (of 0: the least)
        scale = most > 0.f ? power(-inverse) : 1.f;
        if (lane == 0) to.inverse[row] = power(inverse);
    }
#pragma unroll 2
    for (uint32_t k = lane * 8; k < to.ld; k += 256) {
        __align__(16) T v[8];
        eight(k, v);
        if constexpr (kPair) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= scale;
            const uint4 hi = pack8<__half>(v);
            *reinterpret_cast<uint4*>(to.hi + at + k) = hi;
            *reinterpret_cast<uint4*>(to.lo + at + k) = rest8<__half>(v, hi);
        } else {
            *reinterpret_cast<uint4*>(to.hi + at + k) = *reinterpret_cast<uint4*>(v);
        }
    }
    return inverse;
}

// How dh = G W is divided: into parts of the vocabulary side by side, each with a sum of its own.
struct SumPlan {
    uint32_t tiles_n, bm, units;   // tiles of a row of tiles, rows of a tile, CTAs (or pairs) of the GPU
    uint32_t blocks, clocks;       // of k in a piece of the vocabulary; clocks of one
    uint32_t rows;                 // of the sums in all
    static constexpr uint32_t kFixed = 6000, kShortest = 8, kMost = 64;   // clocks of a tile besides; blocks of a part; parts
    // Rows of a part's sum.
    static __host__ __device__ uint32_t part_rows(uint32_t count) { return (count + 31) / 32 * 32; }
    // The parts for `count` kept tokens: those of as many as fill 1 to 4 rounds of the GPU that take the least time.  (3001
    // tokens on 50257 x 1280 of which 900 are kept are 20 tiles for 76 pairs of CTAs: loss and gradient 486 us in one
    // part, 373 in three.)
    __host__ __device__ uint32_t parts(uint32_t count) const {
        const uint32_t tiles = (count + bm - 1) / bm * tiles_n;
        if (tiles == 0) return 1;
        uint32_t most = blocks / kShortest, best = 1;
        if (rows && rows / part_rows(count) < most) most = rows / part_rows(count);
        most = most < 1 ? 1 : most > kMost ? kMost : most;
        uint64_t least = ~uint64_t(0);
        for (uint32_t round = 1; round <= 4; ++round) {
            uint32_t n = round * units / tiles;
            n = n < 1 ? 1 : n > most ? most : n;
            const uint64_t time = uint64_t((tiles * n + units - 1) / units) * ((blocks + n - 1) / n * clocks + kFixed);
            if (time < least) {
                least = time;
                best = n;
            }
        }
        return best;
    }
};

struct GatherArgs {
    const void* h;
    uint64_t h_stride;
    const void* targets;
    int target64;
    int64_t ignore;
    uint32_t tokens, vocab, width, per_block, blocks;
    Planes to;
    const float* grad_loss;   // null, or for `most`: per CTA what Scales::h is the largest of
    uint64_t grad_stride;
    int* most;
    uint32_t* count;          // kept tokens
    uint32_t* splits;         // null, or for SumPlan::parts()
    SumPlan sum;
    int* target;              // per kept row: its target, or -1 if outside the vocabulary
    int* token;               // per kept row: its token
    int* row;                 // per token: its row, or -1
    long long* rest;          // null, or per kept row: set to zero
    uint32_t* status;
    uint32_t gave_up;         // injected_timeout()
};

__device__ __forceinline__ int64_t target_of(const GatherArgs& p, uint32_t t) {
    return p.target64 ? static_cast<const int64_t*>(p.targets)[t] : static_cast<const int32_t*>(p.targets)[t];
}

// Sums of (kept before `first`, kept in all), in every thread.
__device__ __forceinline__ uint2 count_kept(const GatherArgs& p, uint32_t first, uint2* shared) {
    uint2 c = make_uint2(0, 0);
    for (uint32_t t = threadIdx.x; t < p.tokens; t += 256) {
        const uint32_t kept = target_of(p, t) != p.ignore;
        c.y += kept;
        if (t < first) c.x += kept;
    }
    c.x = __reduce_add_sync(0xffffffffu, c.x);
    c.y = __reduce_add_sync(0xffffffffu, c.y);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = c;
    __syncthreads();
    uint2 r = make_uint2(0, 0);
    for (int i = 0; i < 8; ++i) {
        r.x += shared[i].x;
        r.y += shared[i].y;
    }
    return r;
}

// Gathers the kept rows of h in the order of the tokens, and zeros behind them up to a multiple of kRowPad.  Every CTA
// counts all targets itself: that takes 64 KB from L2 for 8192 tokens.
template <typename T>
__device__ __forceinline__ void gather_rows(const GatherArgs& p, int* tops) {
    __shared__ uint2 shared[8];
    const uint32_t first = blockIdx.x * p.per_block, end = min(first + p.per_block, p.tokens);   // (none in the last CTAs of few tokens)
    const uint2 c = count_kept(p, first, shared);
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *p.count = c.y;
        *p.status = p.gave_up;
        if (p.splits) *p.splits = p.sum.parts(c.y);
    }
    uint32_t before = c.x;
    int most = kLeastExponent - 126;
    for (uint32_t t0 = first; t0 < end; t0 += 32) {
        const uint32_t t = t0 + lane;
        const int64_t y = t < end ? target_of(p, t) : p.ignore;
        const uint32_t kept = __ballot_sync(0xffffffffu, y != p.ignore);
        if (warp == 0 && t < end) {
            const uint32_t row = before + __popc(kept & ((1u << lane) - 1));
            p.row[t] = y != p.ignore ? static_cast<int>(row) : -1;
            if (y != p.ignore) {
                p.target[row] = y >= 0 && y < p.vocab ? static_cast<int>(y) : -1;
                p.token[row] = static_cast<int>(t);
                if (p.rest) p.rest[row] = 0;
            }
        }
        uint32_t left = kept;
        for (uint32_t i = 0; left; ++i) {
            const uint32_t at = __ffs(left) - 1;
            left &= left - 1;
            if (i % 8 != warp) continue;
            const T* src = static_cast<const T*>(p.h) + uint64_t(t0 + at) * p.h_stride;
            const int inverse = copy_row(src, p.width, p.to, before + i, lane);
            if (p.grad_loss) {
                const float a = p.grad_loss[(t0 + at) * p.grad_stride];
                if (fabsf(a) < INFINITY) most = max(most, grad_exponent(a) + inverse);
            }
        }
        before += __popc(kept);
    }
    const uint32_t pad = (c.y + kRowPad - 1) / kRowPad * kRowPad;
    for (uint32_t r = c.y + blockIdx.x * 8 + warp; r < pad; r += p.blocks * 8)
        for (uint32_t k = lane * 8; k < p.to.ld; k += 256) {
            *reinterpret_cast<uint4*>(p.to.hi + uint64_t(r) * p.to.ld + k) = uint4{};
            if (p.to.lo) *reinterpret_cast<uint4*>(p.to.lo + uint64_t(r) * p.to.ld + k) = uint4{};
        }
    if (p.most) {
        if (lane == 0) tops[warp] = most;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 1; i < 8; ++i) most = max(most, tops[i]);
            p.most[blockIdx.x] = most;
        }
    }
}

struct PackArgs {
    const void* w;
    uint64_t stride;
    uint32_t rows, width, blocks;
    Planes to;
    int* most;                // per CTA the exponent of the largest inverse scale
};

// W as rows that TMA can read, by `blocks` CTAs.
template <typename T>
__device__ __forceinline__ void pack_rows(const PackArgs& p, uint32_t block, int* tops) {
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    int most = -126;
    for (uint32_t r = block * 8 + warp; r < p.rows; r += p.blocks * 8)
        most = max(most, copy_row(static_cast<const T*>(p.w) + uint64_t(r) * p.stride, p.width, p.to, r, lane));
    if (!p.most) return;
    if (lane == 0) tops[warp] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) most = max(most, tops[i]);
        p.most[block] = most;
    }
}

// The operands of the products: the gathered h and, where W has to be laid out, in further CTAs W.  (One launch for both: f32,
// 509 tokens on 10007 x 451, loss and gradient take 4 us less than with two.)
template <typename T>
__global__ void __launch_bounds__(256) k_ce_operands(const __grid_constant__ GatherArgs h, const __grid_constant__ PackArgs w) {
    __shared__ int tops[8];
    wait_previous();
    if (blockIdx.x < h.blocks) gather_rows<T>(h, tops);
    else pack_rows<T>(w, blockIdx.x - h.blocks, tops);
}

struct EvenArgs {
    const int *most_h, *most_w;
    uint32_t n_h, n_w;
    Scales* scales;
    const uint32_t* count;
    const int* token;
    const float* grad_loss;
    uint64_t grad_stride;
    Planes from, to;          // to.hi: null if not needed
};

// The scales of a call, and grad_loss_t h_t of the gathered rows with one scale for all (zeros behind the kept rows again).
__global__ void __launch_bounds__(256) k_ce_even(const __grid_constant__ EvenArgs p) {
    __shared__ int tops[2];
    if (threadIdx.x < 2) tops[threadIdx.x] = kLeastExponent - 126;
    __syncthreads();
    wait_previous();
    int h = kLeastExponent - 126, w = -126;
    for (uint32_t i = threadIdx.x; i < p.n_h; i += 256) h = max(h, p.most_h[i]);
    if (blockIdx.x == 0)
        for (uint32_t i = threadIdx.x; i < p.n_w; i += 256) w = max(w, p.most_w[i]);
    atomicMax(&tops[0], h);
    atomicMax(&tops[1], w);
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.scales = Scales{tops[0], tops[1]};
    if (!p.to.hi) return;
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, count = *p.count;
    const uint32_t pad = (count + kRowPad - 1) / kRowPad * kRowPad;
    for (uint32_t r = blockIdx.x * 8 + warp; r < pad; r += gridDim.x * 8) {
        float a = 0.f, by = 0.f;   // a: below 2, and half of it by the scale
        if (r < count) {
            a = p.grad_loss[p.token[r] * p.grad_stride];
            const int own = grad_exponent(a), e = own + static_cast<int>(__float_as_uint(p.from.inverse[r]) >> 23) - 127 - tops[0] - 1;
            a *= power(-own);
            by = power(e < -126 ? -126 : e > 0 ? 0 : e);   // (> 0: of a that is not finite)
        }
        for (uint32_t k = lane * 8; k < p.to.ld; k += 256) {
            const uint64_t at = uint64_t(r) * p.to.ld + k;
            const uint4 hi = *reinterpret_cast<const uint4*>(p.from.hi + at), lo = *reinterpret_cast<const uint4*>(p.from.lo + at);
            float v[8];
            unpack8<__half, true>(hi, lo, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] * a * by;
            const uint4 e = pack8<__half>(v);
            *reinterpret_cast<uint4*>(p.to.hi + at) = e;
            *reinterpret_cast<uint4*>(p.to.lo + at) = rest8<__half>(v, e);
        }
    }
}

// The inverse scales of W's rows [col, col + 32), which are columns of the logits.  They are allocated in whole tiles.
__device__ __forceinline__ void scale_columns(float (&v)[32], const float* inverse, uint32_t col, float by) {
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
        const float4 w = *reinterpret_cast<const float4*>(inverse + col + k);
        v[k] *= by * w.x;
        v[k + 1] *= by * w.y;
        v[k + 2] *= by * w.z;
        v[k + 3] *= by * w.w;
    }
}

// Per row and group of COLUMNS of the vocabulary: the largest logit and the sum of 2^(s log2(e) - reference).
template <bool PAIR>
struct EpiLoss {
    static constexpr uint32_t kBuffer = 0;
    const uint32_t* count;
    const int* target;
    const float *h_inverse, *w_inverse;
    float2* partial;          // [groups of columns][rows]
    float* target_logit;      // [rows]
    uint32_t vocab, rows;
    __device__ __forceinline__ void before(const Tile&, uint32_t, uint32_t, const WarpBuffer&) const {}
    template <int COLUMNS, class Columns>
    __device__ __forceinline__ bool tile(const Tile&, uint32_t row, uint32_t col, const Columns& acc, bool, WarpBuffer& buf) const {
        row += buf.lane;
        const bool in = row < *count;
        const int y = in ? target[row] : -1;
        const float by = PAIR && in ? h_inverse[row] : 1.f;
        float top = -INFINITY, sum = 0.f;
#pragma unroll(Columns::kUnroll)
        for (int c = 0; c < COLUMNS; c += 32) {
            const uint32_t c0 = col + c;
            if (c0 >= vocab) break;
            float v[32];
            acc.load(c, v);
            if constexpr (PAIR) scale_columns(v, w_inverse, c0, by);
            if (static_cast<uint32_t>(y) - c0 < 32u) {
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < 32; ++k) s = static_cast<uint32_t>(y) - c0 == k ? v[k] : s;
                target_logit[row] = s;
            }
            if (c0 + 32 > vocab) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] = c0 + k < vocab ? v[k] : -INFINITY;
            }
            float most = v[0];
#pragma unroll
            for (int k = 1; k < 32; ++k) most = fmaxf(most, v[k]);
            most = fmaxf(top, most);
            const float ref = reference(most);
            sum *= rescale(top, ref);
            float part[4] = {};
#pragma unroll
            for (int k = 0; k < 32; ++k) part[k % 4] += exp2_fast(fmaf(v[k], kLog2e, -ref));
            sum += (part[0] + part[1]) + (part[2] + part[3]);
            top = most;
        }
        if (in && col < vocab) partial[uint64_t(col / COLUMNS) * rows + row] = make_float2(top, sum);
        return true;
    }
};

struct JoinArgs {
    const uint32_t* count;
    const int *row, *target, *token;
    const float2* partial;
    const float* target_logit;
    float *loss, *lse;
    uint32_t tokens, groups, rows;
    const uint32_t* status;
};

// Joins the partial results of ROWS rows, in a fixed order: a thread to a row and every kParts'th group of columns.  8 rows to
// a CTA while these run at the same time: bound by the latency of a thread's loads.  (8 and 32 rows: loss of 8 tokens on
// 50257 x 768 21.2 and 23.2 us, of 300 37.5 and 38.9; of 8192 on 5000 x 768 53.8 and 50.3, where a warp's loads are wider
// with 32.)
constexpr uint32_t join_rows(uint32_t tokens) { return tokens <= 8 * kSms ? 8 : 32; }
template <uint32_t ROWS>
__global__ void __launch_bounds__(1024) k_ce_join(const __grid_constant__ JoinArgs p) {
    constexpr uint32_t kParts = 1024 / ROWS;
    __shared__ float2 parts[kParts][ROWS + 1];
    wait_previous();
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, count = *p.count;
    const uint32_t own = threadIdx.x % ROWS, part = threadIdx.x / ROWS;
    uint32_t r = blockIdx.x * ROWS + own;
    float2 v = make_float2(-INFINITY, 0.f);
    if (r < count) {
#pragma unroll 8
        for (uint32_t i = part; i < p.groups; i += kParts) v = joined(v, p.partial[uint64_t(i) * p.rows + r]);
    }
    parts[part][own] = v;
    const bool failed = *p.status != 0;   // partial results are missing: all is NaN
    if (part == 0 && r < p.tokens && (failed || p.row[r] < 0)) p.loss[r] = p.lse[r] = failed ? NAN : 0.f;
    __syncthreads();
    // a warp to a row: its parts
    if (warp >= ROWS) return;
    r = blockIdx.x * ROWS + warp;
    v = parts[lane][warp];
    for (uint32_t i = lane + 32; i < kParts; i += 32) v = joined(v, parts[i][warp]);
    for (int o = 16; o; o >>= 1)
        v = joined(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
    if (lane || r >= count || failed) return;
    const bool known = p.target[r] >= 0;   // else a target outside the vocabulary
    const float lse = known ? log_sum(v) : NAN;
    p.lse[p.token[r]] = lse;
    p.loss[p.token[r]] = lse - p.target_logit[r];
}

// What a row of the rounded G adds up to is kept as a whole number, so that the order of the additions does not matter: in units
// of 2^-kRestBits times grad_loss' power of two, so that grad_loss itself is below 2^(kRestBits + 1).
constexpr int kRestBits = 40;

// A piece of G from the logits.  Rows beyond the kept ones are written as zeros: the products over G read them.  With PAIR
// it is written twice, scaled for dh and for dW.
template <bool PAIR>
struct EpiGrad {
    static constexpr uint32_t kBuffer = 4096;
    CUtensorMap to[PAIR ? 4 : 1];   // G, the piece's columns; PAIR: hi and lo for dh, then for dW
    const uint32_t* count;
    const int *target, *token;
    const float *lse, *grad_loss, *h_inverse, *w_inverse;
    const Scales* scales;
    long long* rest;          // 16-bit: per row what its rounded G adds up to, see kRestBits
    uint64_t grad_stride;
    uint32_t v0, columns;     // the piece's first vocabulary row and their number
    int for_h, for_w;         // which of G's forms are needed
    __device__ __forceinline__ void before(const Tile&, uint32_t, uint32_t, const WarpBuffer&) const {}
    template <int COLUMNS, class Columns>
    __device__ __forceinline__ bool tile(const Tile&, uint32_t row, uint32_t col, const Columns& acc, bool, WarpBuffer& buf) const {
        const bool in = row + buf.lane < *count;
        uint32_t y = 0xffffffffu;
        float a = 0.f, ref = 0.f, by = 1.f;
        if (in) {
            const uint32_t tok = token[row + buf.lane];
            y = static_cast<uint32_t>(target[row + buf.lane]) - v0;
            ref = PAIR ? lse[tok] : lse[tok] * kLog2e;
            if constexpr (PAIR) by = h_inverse[row + buf.lane];
            else a = grad_loss[tok * grad_stride];
        }
        float left[2] = {};
#pragma unroll
        for (int c = 0; c < COLUMNS; c += 64) {
            const uint32_t c0 = col + c;
            float v[64];
            acc.load(c, *reinterpret_cast<float(*)[32]>(v));
            acc.load(c + 32, *reinterpret_cast<float(*)[32]>(v + 32));
            if (c + 64 == COLUMNS) acc.done();
            if (c0 >= columns) continue;
            const float* iw = PAIR ? w_inverse + v0 + c0 : nullptr;
#pragma unroll
            for (int k = 0; k < 64; ++k) {
                // (32-bit: the difference first, which is exact where the probability is large)
                float g = exp2_fast(PAIR ? (v[k] * (by * iw[k]) - ref) * kLog2e : fmaf(v[k], kLog2e, -ref));
                if (y - c0 == k) g -= 1.f;
                v[k] = !in ? 0.f : PAIR ? g : g * a;
            }
            auto store = [&](const CUtensorMap& map, auto piece) {
                buf.reuse();
#pragma unroll
                for (int j = 0; j < 8; ++j) sts128(buf.at(j), piece(j));
                if (buf.written()) {
                    tma_store(&map, buf.addr, c0, row, 0);
                    tma_store_commit();
                }
            };
            if constexpr (!PAIR) {
                if (c0 + 64 > columns) {   // (what lies beyond is not stored)
#pragma unroll
                    for (int k = 0; k < 64; ++k) v[k] = c0 + k < columns ? v[k] : 0.f;
                }
                store(to[0], [&](int j) {
                    const uint4 e = pack8<__nv_bfloat16>(v + 8 * j);
                    const uint32_t words[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = unpack<__nv_bfloat16>(words[i]);
                        left[0] += f.x;
                        left[1] += f.y;
                    }
                    return e;
                });
            } else {
                auto both = [&](int first, auto value) {
                    auto eight = [&](int j, float (&x)[8]) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = value(8 * j + i);
                    };
                    float x[8];
                    store(to[first], [&](int j) {
                        eight(j, x);
                        return pack8<__half>(x);
                    });
                    store(to[first + 1], [&](int j) {
                        eight(j, x);
                        return rest8<__half>(x, pack8<__half>(x));
                    });
                };
                // |G_tv| <= 1: with 2^kTopExponent below f16's range
                const float down = power(-scales->w), up = power(kTopExponent);
                if (for_h) both(0, [&](int k) { return v[k] * up * (iw[k] * down); });
                if (for_w) both(2, [&](int k) { return v[k] * up; });
            }
        }
        if (!PAIR && in && for_h && col < columns)
            atomicAdd(reinterpret_cast<unsigned long long*>(rest + row + buf.lane),
                      static_cast<unsigned long long>(__float2ll_rn(times_power(left[0] + left[1], kRestBits - exponent(a)))));
        return true;
    }
};

// dh's sums: [split][rows][ld] in f32.
struct EpiSum {
    static constexpr uint32_t kBuffer = 4096;
    CUtensorMap to;           // the parts' sums one below another
    const uint32_t* count;
    uint32_t ld;
    int add;                  // to what the pieces before have left
    __device__ __forceinline__ void before(const Tile&, uint32_t, uint32_t, const WarpBuffer&) const {}
    template <int COLUMNS, class Columns>
    __device__ __forceinline__ bool tile(const Tile& t, uint32_t row, uint32_t col, const Columns& acc, bool empty, WarpBuffer& buf) const {
        const bool any = row < *count;
        const uint32_t y = t.split * SumPlan::part_rows(*count) + row;
#pragma unroll(Columns::kUnroll)
        for (int c = 0; c < COLUMNS; c += 32) {
            float v[32];
            if (col + c >= ld || !any) break;
            acc.load(c, v);
            if (add && empty) continue;
            buf.reuse();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float4 x = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                if (empty) x = make_float4(0.f, 0.f, 0.f, 0.f);
                sts128(buf.at(j), *reinterpret_cast<uint4*>(&x));
            }
            if (buf.written()) {
                if (add) tma_add(&to, buf.addr, col + c, y, 0);
                else tma_store(&to, buf.addr, col + c, y, 0);
                tma_store_commit();
            }
        }
        return true;
    }
};

// A piece's rows of dW.
template <typename T>
struct EpiWeight {
    static constexpr uint32_t kBuffer = 4096;
    CUtensorMap to;           // of the piece's rows, if tma
    T* dw;                    // of the piece's first row
    uint64_t stride;
    const Scales* scales;     // of 32-bit operands
    uint32_t rows, width;
    int tma;
    __device__ __forceinline__ void before(const Tile&, uint32_t, uint32_t, const WarpBuffer&) const {}
    template <int COLUMNS, class Columns>
    __device__ __forceinline__ bool tile(const Tile&, uint32_t row, uint32_t col, const Columns& acc, bool empty, WarpBuffer& buf) const {
        constexpr bool kPair = sizeof(T) == 4;
        constexpr int kBox = 128 / sizeof(T), kPer = 16 / sizeof(T);
        const int e = kPair ? scales->h + 1 - kTopExponent : 0;
        const float by[2] = {power(e / 2), power(e - e / 2)};
#pragma unroll
        for (int c = 0; c < COLUMNS; c += kBox) {
            float v[kBox];
#pragma unroll
            for (int k = 0; k < kBox; k += 32) acc.load(c + k, *reinterpret_cast<float(*)[32]>(v + k));
            if (c + kBox == COLUMNS) acc.done();
            if (row >= rows || col + c >= width) continue;
            buf.reuse();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint4 r;
                if constexpr (kPair)
                    r = make_uint4(__float_as_uint(v[4 * j] * by[0] * by[1]), __float_as_uint(v[4 * j + 1] * by[0] * by[1]),
                                   __float_as_uint(v[4 * j + 2] * by[0] * by[1]), __float_as_uint(v[4 * j + 3] * by[0] * by[1]));
                else
                    r = pack8<T>(v + kPer * j);
                sts128(buf.at(j), empty ? uint4{} : r);
            }
            if (tma && ends_whole<T>(col + c + kBox, width)) {
                if (buf.written()) {
                    tma_store(&to, buf.addr, col + c, row, 0);
                    tma_store_commit();
                }
            } else {
                __syncwarp();
                store_box(buf.addr, buf.lane, dw + row * stride + col + c, stride, 1, rows - row, width - (col + c));
                __syncwarp();
            }
        }
        return true;
    }
};

struct ScatterArgs {
    const int *row, *target;
    const float *sum, *grad_loss;
    const Scales* scales;     // of 32-bit operands
    uint64_t grad_stride;
    const uint32_t *count, *splits;
    const long long* rest;    // of 16-bit operands
    const void* w;
    uint64_t stride, w_stride;
    uint32_t ld, tokens, width;
    void* dh;
    const uint32_t* status;
    void* dw;                 // null, or to be made NaN with dh after a wait that ran out
    uint64_t dw_stride;
    uint32_t vocab;
};

// dh from the sums, back in the order of the tokens; zeros for the ignored ones.  16-bit: without what the rounding of G has left
// of its rows' sums, which goes to the target's row of W.  128 columns of a token are taken by one
// warp, or with MANY parts by a CTA, whose 8 warps have every 8th part each (64 tokens, 50 parts: 16 us by single warps).
template <typename T, bool MANY>
__global__ void __launch_bounds__(256) k_ce_scatter(const __grid_constant__ ScatterArgs p) {
    __shared__ float4 parts[8][32];
    wait_previous();
    if (*p.status) {
        const uint64_t me = uint64_t(blockIdx.x) * 256 + threadIdx.x, all = uint64_t(gridDim.x) * 256;
        if (p.dh) fill_nan(static_cast<T*>(p.dh), 1, p.tokens, p.width, 0, p.stride, 1, me, all);
        if (p.dw) fill_nan(static_cast<T*>(p.dw), 1, p.vocab, p.width, 0, p.dw_stride, 1, me, all);
        return;
    }
    if (!p.dh) return;
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, per_row = (p.width + 127) / 128;
    const bool vec = p.stride % 4 == 0 && reinterpret_cast<uintptr_t>(p.dh) % (4 * sizeof(T)) == 0;
    const uint32_t splits = *p.splits;
    const uint64_t plane = uint64_t(SumPlan::part_rows(*p.count)) * p.ld;
    const uint64_t first = MANY ? blockIdx.x : uint64_t(blockIdx.x) * 8 + warp, step = MANY ? gridDim.x : uint64_t(gridDim.x) * 8;
    for (uint64_t i = first; i < uint64_t(p.tokens) * per_row; i += step) {
        const uint32_t t = static_cast<uint32_t>(i / per_row), c = static_cast<uint32_t>(i % per_row) * 128 + lane * 4;
        const int row = p.row[t];
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float4& x) {
            v.x += x.x;
            v.y += x.y;
            v.z += x.z;
            v.w += x.w;
        };
        if (row >= 0 && c < p.width) {
            const float* at = p.sum + uint64_t(row) * p.ld + c;
#pragma unroll 4
            for (uint32_t s = MANY ? warp : 0; s < splits; s += MANY ? 8 : 1) add(*reinterpret_cast<const float4*>(at + s * plane));
        }
        if constexpr (MANY) {
            __syncthreads();   // the last token's parts have been read
            parts[warp][lane] = v;
            __syncthreads();
            if (warp) continue;
            for (int k = 1; k < 8; ++k) add(parts[k][lane]);
        }
        if (c >= p.width) continue;
        if constexpr (sizeof(T) == 2) {
            const int y = row >= 0 ? p.target[row] : -1;
            if (y >= 0) {
                const float rest = times_power(__ll2float_rn(p.rest[row]), exponent(p.grad_loss[t * p.grad_stride]) - kRestBits);
                const T* at = static_cast<const T*>(p.w) + uint64_t(y) * p.w_stride + c;
                float x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = c + k < p.width ? to_float(at[k]) : 0.f;
                v = make_float4(fmaf(-rest, x[0], v.x), fmaf(-rest, x[1], v.y), fmaf(-rest, x[2], v.z), fmaf(-rest, x[3], v.w));
            }
        } else {
            if (row >= 0) {
                float a = p.grad_loss[t * p.grad_stride];
                const int own = grad_exponent(a), e = own + p.scales->w - kTopExponent;
                a *= power(-own);
                v = make_float4(times_power(v.x * a, e), times_power(v.y * a, e), times_power(v.z * a, e), times_power(v.w * a, e));
            }
        }
        __align__(16) T out[4] = {round_to<T>(v.x), round_to<T>(v.y), round_to<T>(v.z), round_to<T>(v.w)};
        T* at = static_cast<T*>(p.dh) + t * p.stride + c;
        if (vec && c + 4 <= p.width) {
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(at) = *reinterpret_cast<uint2*>(out);
            else *reinterpret_cast<uint4*>(at) = *reinterpret_cast<uint4*>(out);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c + k < p.width) at[k] = out[k];
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

// Tiles of the products: 256 columns, or 128 where the sums are held in registers (32-bit operands).
template <bool PAIR>
constexpr int kTileN = PAIR ? 128 : 256;
// k between two additions to sums in registers.  16-bit operands: 512 in the logits, if there are more at all (what the
// accumulators cut off of 1600 k reaches 1e-6 of the loss).  32-bit ones: 64 in all products, one stage, whose terms with lo
// come first, while the sum is small.  Then errors are below those of f32 arithmetic (loss, lse, dh and dW of 509 tokens on
// 10007 x 451: 1.4e-7, 8e-8, 2.9e-7, 2.8e-7, and twice that with 128 in the logits); loss and gradient of these take 127.5 us
// and 125.5, of 1024 tokens on 50257 x 768 776 and 733.
constexpr uint32_t kUnchunked = 512;
template <bool PAIR>
constexpr uint32_t kChunk = PAIR ? 64 : 512;
constexpr int kPairRows = 128;                   // up to so many tokens a CTA multiplies by itself (CG = 1), else pairs do
constexpr int kPieceUnit = 256;                  // pieces of the vocabulary come in multiples of this
constexpr uint64_t kPieceBytes = 256ull << 20;   // most bytes of a piece of G with 16-bit operands, half of them with 32-bit ones

constexpr uint32_t kGatherBlocks = 512, kPackBlocks = 2048;   // most CTAs of those kernels

// Few tokens go another way (few_tokens.cuh), if their rows of h fit into shared memory: up to 4 with 16-bit operands, up
// to 16 with 32-bit ones, which the products would have to lay out first.  This way and by the products, vocabulary 50257 x
// 768: loss of 4 tokens bf16 24 and 28 us, of 8 35 and 27, of 16 f32 61 and 87, of 32 114 and 88; loss and gradient of 4
// tokens bf16 83 and 89 us, of 8 129 and 89, of 16 f32 210 and 259.  (Where W has to be laid out because of its alignment,
// x 1102, 5 to 8 tokens bf16: loss 72 and 83, loss and gradient 232 and 221: no rule of its own.)
constexpr uint32_t kFew16 = 4, kFew32 = 16, kFewSmem = 208 * 1024;
int few_size(const dsm_linear_ce& p) {   // tokens of the kernels' variant; 0: not few
    if (p.tokens == 0 || p.tokens > (p.dtype == DSM_F32 ? kFew32 : kFew16)) return 0;
    const int tn = p.tokens <= 1 ? 1 : p.tokens <= 4 ? 4 : p.tokens <= 8 ? 8 : 16;
    const uint32_t padded = p.dtype == DSM_F32 ? few_padded<float>(p.width) : few_padded<__nv_bfloat16>(p.width);
    return uint64_t(tn) * padded * 4 <= kFewSmem ? tn : 0;
}

struct Plan {
    int few;                  // few_size()
    float *few_g, *few_sum;
    uint32_t few_splits;
    uint32_t rows;            // tokens, padded
    int tile_v;               // columns of a tile of the logits
    uint32_t groups;          // of the vocabulary's columns, each with a partial result of the loss
    bool pair, pack;          // 32-bit operands; W has to be laid out for TMA
    Planes h, w, even;        // even: grad_loss_t h_t with one scale for all rows
    uint16_t* g[4];           // hi; hi and lo for dh, for dW
    uint32_t* count;          // kept tokens; parts of dh
    int *target, *token, *row;
    long long* rest;
    float2* partial;
    float* target_logit;
    int *most_h, *most_w;
    Scales* scales;
    uint32_t piece, pieces;   // vocabulary rows of a piece of G
    SumPlan parts;            // of dh
    uint32_t splits, ld_sum;  // splits: parts if all tokens are kept
    float* sum;
    uint64_t bytes;
};

Plan make_plan(const dsm_linear_ce& p, bool grad, void* workspace) {
    Plan r{};
    r.rows = static_cast<uint32_t>(round_up(p.tokens ? p.tokens : 1, kRowPad));
    r.pair = p.dtype == DSM_F32;
    r.tile_v = r.pair ? kTileN<true> : kTileN<false>;
    // With one row of tiles the vocabulary has few rounds of the SMs: half as wide tiles where they fill them better
    // (50257 rows: 3 rounds of 128 for 2 of 256).
    if (!r.pair && p.tokens <= kPairRows && ceil_div(ceil_div(p.vocab, 128), kSms) < 2 * ceil_div(ceil_div(p.vocab, 256), kSms))
        r.tile_v = 128;
    r.groups = ceil_div(p.vocab, r.tile_v / 2);   // an epilogue warp has half a tile's columns
    r.pack = r.pair || !mappable(p.w, static_cast<int64_t>(p.w_stride), 16, p.vocab, 1, 2);
    r.h.ld = r.w.ld = static_cast<uint32_t>(round_up(p.width, 8));
    Carver c(workspace);
    if ((r.few = few_size(p))) {
        r.ld_sum = static_cast<uint32_t>(round_up(p.width, 32));
        if (grad) {
            // rows of W in as many parts as keep the SMs at work twice over, of at least 32 rows
            const uint32_t columns = r.pair ? few_columns<float>(r.few) : few_columns<__nv_bfloat16>(r.few);
            const uint32_t blocks = ceil_div(p.width, kOuterThreads * columns), parts = ceil_div(3 * kSms, blocks);
            r.few_splits = parts < ceil_div(p.vocab, 32) ? parts : ceil_div(p.vocab, 32);
            r.few_g = c.take<float>(uint64_t(p.vocab) * r.few);
            r.few_sum = c.take<float>(uint64_t(r.few_splits) * r.few * r.ld_sum);
        } else {
            r.partial = c.take<float2>(uint64_t(kSms) * 4 * r.few);
            r.target_logit = c.take<float>(r.few);
        }
        r.bytes = c.used;
        return r;
    }
    r.count = c.take<uint32_t>(2);
    r.target = c.take<int>(r.rows);
    r.token = c.take<int>(r.rows);
    r.row = c.take<int>(r.rows);
    r.h.hi = c.take<uint16_t>(uint64_t(r.rows) * r.h.ld);
    if (r.pack) r.w.hi = c.take<uint16_t>(uint64_t(p.vocab) * r.w.ld);
    if (r.pair) {
        r.h.lo = c.take<uint16_t>(uint64_t(r.rows) * r.h.ld);
        r.w.lo = c.take<uint16_t>(uint64_t(p.vocab) * r.w.ld);
        r.h.inverse = c.take<float>(r.rows);
        r.w.inverse = c.take<float>(round_up(p.vocab, kPieceUnit));
        r.most_h = c.take<int>(kGatherBlocks);
        r.most_w = c.take<int>(kPackBlocks);
        r.scales = c.take<Scales>(1);
    }
    if (!grad) {
        r.partial = c.take<float2>(uint64_t(r.groups) * r.rows);
        r.target_logit = c.take<float>(r.rows);
    } else {
        // a whole number of units, so that rounding up to one does not pass the bound (but one at least)
        const uint64_t all = round_up(p.vocab, kPieceUnit), fit = kPieceBytes / ((r.pair ? 4 : 2) * uint64_t(r.rows));
        const uint64_t most = fit < kPieceUnit ? kPieceUnit : fit / kPieceUnit * kPieceUnit;
        r.pieces = most >= all ? 1 : ceil_div(all, most);
        r.piece = static_cast<uint32_t>(round_up(ceil_div(all, r.pieces), kPieceUnit));
        r.pieces = ceil_div(p.vocab, r.piece);
        if (!r.pair) r.rest = c.take<long long>(r.rows);
        for (int i = 0; i < (r.pair ? 4 : 1); ++i) r.g[i] = c.take<uint16_t>(uint64_t(r.rows) * r.piece);
        if (r.pair) {
            r.even.ld = r.h.ld;
            r.even.hi = c.take<uint16_t>(uint64_t(r.rows) * r.h.ld);
            r.even.lo = c.take<uint16_t>(uint64_t(r.rows) * r.h.ld);
        }
        r.ld_sum = static_cast<uint32_t>(round_up(p.width, 32));
        const uint32_t cg = p.tokens > kPairRows ? 2 : 1, tile_n = r.pair ? kTileN<true> : kTileN<false>;
        r.parts = SumPlan{ceil_div(p.width, tile_n), 128 * cg, kSms / cg, r.piece / kBlockK, tile_n * (r.pair ? 3 : 1), 0};
        r.splits = r.parts.parts(p.tokens);
        // as many rows as that takes, or as one round takes with fewer kept tokens
        const uint32_t round = r.parts.units / r.parts.tiles_n * r.parts.bm, all_rows = r.splits * SumPlan::part_rows(p.tokens ? p.tokens : 1);
        r.parts.rows = round > all_rows ? round : all_rows;
        r.sum = c.take<float>(uint64_t(r.parts.rows) * r.ld_sum);
    }
    r.bytes = c.used;
    return r;
}

int check_args(const char* func, const dsm_linear_ce* p) {
    if (!p) return fail(func, DSM_EINVAL, "NULL argument");
    if (p->dtype != DSM_F32 && p->dtype != DSM_BF16) return fail(func, DSM_EINVAL, "dtype %d unknown", p->dtype);
    if (p->target_bytes != 4 && p->target_bytes != 8) return fail(func, DSM_EINVAL, "target_bytes must be 4 or 8");
    if (p->reserved) return fail(func, DSM_EINVAL, "reserved must be 0");
    if (p->vocab == 0 || p->width == 0) return fail(func, DSM_EINVAL, "vocab and width must be >= 1");
    if (p->tokens > 1u << 24 || p->vocab > 1u << 24 || p->width > 1u << 20)
        return fail(func, DSM_ERANGE, "at most 2^24 tokens, 2^24 vocabulary rows and a width of 2^20");
    if (p->h_stride < p->width && p->tokens > 1) return fail(func, DSM_EINVAL, "h_stride must be >= width");
    if (p->w_stride < p->width && p->vocab > 1) return fail(func, DSM_EINVAL, "w_stride must be >= width");
    return DSM_OK;
}

// The vectors of f32, one value per token.
int check_vectors(const char* func, const dsm_linear_ce& p, const void* a, const void* b, const char* names) {
    if (p.tokens && (reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) % 4)
        return fail(func, DSM_EALIGN, "%s must be aligned to their elements", names);
    return DSM_OK;
}

template <typename T>
cudaError_t gather(const dsm_linear_ce& p, const Plan& r, const float* grad_loss, uint64_t grad_stride, bool for_w,
                   uint32_t* status, cudaStream_t s) {
    GatherArgs a{};
    a.h = p.h;
    a.h_stride = p.h_stride;
    a.targets = p.targets;
    a.target64 = p.target_bytes == 8;
    a.ignore = p.ignore_index;
    a.tokens = p.tokens;
    a.vocab = p.vocab;
    a.width = p.width;
    a.to = r.h;
    a.count = r.count;
    if (grad_loss) {
        a.splits = r.count + 1;
        a.sum = r.parts;
        a.rest = r.rest;
    }
    a.target = r.target;
    a.token = r.token;
    a.row = r.row;
    a.status = status;
    a.gave_up = injected_timeout();
    const bool scaled = r.pair && grad_loss;
    if (scaled) {
        a.grad_loss = grad_loss;
        a.grad_stride = grad_stride;
        a.most = r.most_h;
    }
    a.per_block = ceil_div(p.tokens, kGatherBlocks) < 8 ? 8 : ceil_div(p.tokens, kGatherBlocks);
    // at least 32: they zero the rows behind the kept ones as well (one CTA takes 6 us for 248 rows)
    const uint32_t needed = ceil_div(p.tokens, a.per_block);
    a.blocks = needed < 32 ? 32 : needed;
    PackArgs k{};
    if (r.pack) {
        const uint32_t most = ceil_div(p.vocab, 8);
        k = PackArgs{p.w, p.w_stride, p.vocab, p.width, most < kPackBlocks ? most : kPackBlocks, r.w, scaled ? r.most_w : nullptr};
    }
    const cudaError_t err = launch_grid(k_ce_operands<T>, dim3(a.blocks + k.blocks), 256, 0, s, a, k);
    if (err != cudaSuccess || !scaled) return err;
    Planes even = r.even;
    if (!for_w) even.hi = even.lo = nullptr;
    return launch_grid(k_ce_even, dim3(for_w ? a.blocks : 1), 256, 0, s,
                       EvenArgs{r.most_h, r.most_w, a.blocks, k.blocks, r.scales, r.count, r.token, grad_loss, grad_stride, r.h, even});
}

// Arguments that both calls check against the device.
int check_call(const char* func, const dsm_linear_ce* p, const Plan& r, void* workspace, size_t workspace_bytes, int dev) {
    if (!p->w || !workspace || (p->tokens && (!p->h || !p->targets))) return fail(func, DSM_EINVAL, "NULL argument");
    const uintptr_t esize = p->dtype == DSM_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(p->h) % esize || reinterpret_cast<uintptr_t>(p->w) % esize ||
        reinterpret_cast<uintptr_t>(p->targets) % p->target_bytes)
        return fail(func, DSM_EALIGN, "h, w and targets must be aligned to their elements");
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return fail(func, DSM_EALIGN, "the workspace must be 256-byte aligned");
    if (workspace_bytes < r.bytes)
        return fail(func, DSM_ENOMEM, "the workspace has %zu bytes, %llu are needed", workspace_bytes,
                    static_cast<unsigned long long>(r.bytes));
    if (int rc = check_device(func, workspace, "workspace", dev)) return rc;
    if (int rc = check_device(func, p->w, "w", dev)) return rc;
    if (p->tokens) {
        if (int rc = check_device(func, p->h, "h", dev)) return rc;
        if (int rc = check_device(func, p->targets, "targets", dev)) return rc;
    }
    return DSM_OK;
}

// W (or its packed form) from row v0 on, as an operand whose box has `rows` rows.
int weight_maps(const char* func, const dsm_linear_ce& p, const Plan& r, uint32_t v0, uint32_t count, uint32_t rows,
                CUtensorMap (&maps)[2]) {
    for (int i = 0; i < 2; ++i) {
        const uint16_t* base = !r.pack ? static_cast<const uint16_t*>(p.w) : i && r.pair ? r.w.lo : r.w.hi;
        const uint64_t ld = r.pack ? r.w.ld : p.w_stride;
        if (int rc = make_map(func, &maps[i], base + uint64_t(v0) * ld, p.width, count, 1, ld, 0, rows,
                              r.pair ? Elem::f16 : Elem::bf16))
            return rc;
    }
    return DSM_OK;
}

int hidden_maps(const char* func, const dsm_linear_ce& p, const Plan& r, const Planes& h, uint32_t rows, CUtensorMap (&maps)[2]) {
    for (int i = 0; i < 2; ++i)
        if (int rc = make_map(func, &maps[i], i && r.pair ? h.lo : h.hi, p.width, r.rows, 1, h.ld, 0, rows,
                              r.pair ? Elem::f16 : Elem::bf16))
            return rc;
    return DSM_OK;
}

FewArgs few_args(const dsm_linear_ce& p, const Plan& r, uint32_t* status) {
    FewArgs a{};
    a.h = p.h;
    a.w = p.w;
    a.targets = p.targets;
    a.h_stride = p.h_stride;
    a.w_stride = p.w_stride;
    a.ignore = p.ignore_index;
    a.tokens = p.tokens;
    a.vocab = p.vocab;
    a.width = p.width;
    a.target64 = p.target_bytes == 8;
    const int esize = p.dtype == DSM_BF16 ? 2 : 4;
    a.vec = reinterpret_cast<uintptr_t>(p.w) % 16 == 0 && (p.vocab == 1 || p.w_stride * esize % 16 == 0);
    a.status = status;
    a.partial = r.partial;
    a.target_logit = r.target_logit;
    a.g = r.few_g;
    a.sum = r.few_sum;
    a.ld = r.ld_sum;
    a.splits = r.few_splits;
    return a;
}

template <typename T, int TN, bool GRAD>
cudaError_t few_logits(const FewArgs& a, int sms, uint32_t* ctas, cudaStream_t s) {
    constexpr int R = TN <= 4 ? 8 : 4, kFewThreads = few_threads(R * TN);
    auto kernel = k_ce_few<T, TN, R, GRAD>;
    const size_t smem = TN * few_padded<T>(a.width) * 4;
    const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    if (err != cudaSuccess) return err;
    const uint32_t want = ceil_div(a.vocab, R * (kFewThreads / 32)), most = sms < 4 * static_cast<int>(kSms) ? sms : 4 * kSms;
    *ctas = want < most ? want : most;
    return launch_grid(kernel, dim3(*ctas), kFewThreads, smem, s, a);
}

template <typename T, int TN>
cudaError_t few_loss(const FewArgs& a, int sms, cudaStream_t s) {
    uint32_t ctas = 0;
    const cudaError_t err = few_logits<T, TN, false>(a, sms, &ctas, s);
    return err != cudaSuccess ? err : launch_grid(k_ce_few_join<TN>, dim3(1), 32 * TN, 0, s, a, ctas);
}

template <typename T, int TN>
cudaError_t few_grad(const FewArgs& a, int sms, cudaStream_t s) {
    constexpr int C = few_columns<T>(TN);
    uint32_t ctas = 0;
    cudaError_t err = few_logits<T, TN, true>(a, sms, &ctas, s);
    if (err != cudaSuccess) return err;
    constexpr int kApart = C > 4 ? 4 : C;   // (a register each)
    err = a.vec && a.out_vec
              ? launch_grid(k_ce_few_outer<T, TN, C, true>, dim3(ceil_div(a.width, kOuterThreads * C), a.splits), kOuterThreads, 0, s, a)
              : launch_grid(k_ce_few_outer<T, TN, kApart, false>, dim3(ceil_div(a.width, kOuterThreads * kApart), a.splits),
                            kOuterThreads, 0, s, a);
    return err != cudaSuccess || !a.dh ? err : launch_grid(k_ce_few_sum<T, TN>, dim3(ceil_div(a.width, 32), a.tokens), 1024, 0, s, a);
}

template <typename T>
cudaError_t few(const FewArgs& a, int size, bool grad, int sms, cudaStream_t s) {
    if (size == 1) return grad ? few_grad<T, 1>(a, sms, s) : few_loss<T, 1>(a, sms, s);
    if constexpr (sizeof(T) == 4) {
        if (size == 8) return grad ? few_grad<T, 8>(a, sms, s) : few_loss<T, 8>(a, sms, s);
        if (size == 16) return grad ? few_grad<T, 16>(a, sms, s) : few_loss<T, 16>(a, sms, s);
    }
    return grad ? few_grad<T, 4>(a, sms, s) : few_loss<T, 4>(a, sms, s);
}

// The partial results of the loss.
template <bool PAIR, int CG, int BN = kTileN<PAIR>>
int forward(const char* func, const dsm_linear_ce& p, const Plan& r, uint32_t* status, int sms, cudaStream_t s) {
    constexpr int kTerms = PAIR ? 3 : 1;
    Maps maps;
    if (int rc = hidden_maps(func, p, r, r.h, 128, maps.a)) return rc;
    if (int rc = weight_maps(func, p, r, 0, p.vocab, BN / CG, maps.b)) return rc;
    Schedule w{};
    w.batches = w.splits = 1;
    w.status = status;
    w.tiles_m = ceil_div(p.tokens, 128 * CG);
    w.tiles_n = ceil_div(p.vocab, BN);
    w.k = p.width;
    w.m_count = r.count;
    EpiLoss<PAIR> e{r.count, r.target, r.h.inverse, r.w.inverse, r.partial, r.target_logit, p.vocab, r.rows};
    const uint64_t tiles = uint64_t(w.tiles_m) * w.tiles_n;
    cudaError_t err;
    if (PAIR || w.k > kUnchunked) err = launch_gemm<CG, BN, kTerms, kChunk<PAIR>, !PAIR, false, false>(maps, w, e, tiles, sms, s);
    else err = launch_gemm<CG, BN, kTerms, PAIR ? kChunk<PAIR> : 0, !PAIR, false, false>(maps, w, e, tiles, sms, s);
    return err == cudaSuccess ? DSM_OK : cuda_fail(func, err, "launch the logits");
}

template <bool PAIR, int CG, int BV = kTileN<PAIR>>
int backward(const char* func, const dsm_linear_ce& p, const Plan& r, const float* lse, const float* grad_loss,
             uint64_t grad_stride, void* dh, uint64_t dh_stride, void* dw, uint64_t dw_stride, uint32_t* status, int sms,
             cudaStream_t s) {
    using T = std::conditional_t<PAIR, float, __nv_bfloat16>;
    constexpr int BN = kTileN<PAIR>, kTerms = PAIR ? 3 : 1;
    constexpr Elem kElem = PAIR ? Elem::f16 : Elem::bf16, kOut = PAIR ? Elem::f32 : Elem::bf16;
    cudaError_t err;
    Schedule base{};
    base.batches = 1;
    base.splits = 1;
    base.status = status;
    CUtensorMap hk[2], hm[2];
    if (int rc = hidden_maps(func, p, r, r.h, 128, hk)) return rc;
    if (int rc = hidden_maps(func, p, r, r.pair ? r.even : r.h, 64, hm)) return rc;
    EpiSum es{{}, r.count, r.ld_sum, 0};
    if (int rc = make_map(func, &es.to, r.sum, r.ld_sum, r.parts.rows, 1, r.ld_sum, 0, 32, Elem::f32)) return rc;
    for (uint32_t i = 0; i < r.pieces; ++i) {
        const uint32_t v0 = i * r.piece, count = p.vocab - v0 < r.piece ? p.vocab - v0 : r.piece;
        CUtensorMap gk[2], gm[2], wk[2], wm[2];
        if (int rc = weight_maps(func, p, r, v0, count, BV / CG, wk)) return rc;
        if (int rc = weight_maps(func, p, r, v0, count, 64, wm)) return rc;
        EpiGrad<PAIR> eg{{},        r.count,  r.target,    r.token, lse,   grad_loss,     r.h.inverse,
                         r.w.inverse, r.scales, r.rest,      grad_stride, v0,  count, dh != nullptr, dw != nullptr};
        for (int k = 0; k < 2; ++k) {
            const uint16_t *for_h = r.g[PAIR ? k : 0], *for_w = r.g[PAIR ? 2 + k : 0];
            if (int rc = make_map(func, &gk[k], for_h, count, r.rows, 1, r.piece, 0, 128, kElem)) return rc;
            if (int rc = make_map(func, &gm[k], for_w, count, r.rows, 1, r.piece, 0, 64, kElem)) return rc;
            if (!PAIR && k) break;
            if (int rc = make_map(func, &eg.to[k], for_h, count, r.rows, 1, r.piece, 0, 32, kElem)) return rc;
            if constexpr (PAIR)
                if (int rc = make_map(func, &eg.to[2 + k], for_w, count, r.rows, 1, r.piece, 0, 32, kElem)) return rc;
        }
        // the piece of G
        Schedule w = base;
        w.tiles_m = ceil_div(p.tokens, 128 * CG);
        w.tiles_n = ceil_div(count, BV);
        w.k = p.width;
        w.m_count = r.count;
        const Maps logits{{hk[0], hk[1]}, {wk[0], wk[1]}};
        const uint64_t tiles = uint64_t(w.tiles_m) * w.tiles_n;
        // (as the loss forms them: what is cut off then cancels against lse, and a sure token's p - 1 is right)
        if (PAIR || w.k > kUnchunked) err = launch_gemm<CG, BV, kTerms, kChunk<PAIR>, !PAIR, false, false>(logits, w, eg, tiles, sms, s);
        else err = launch_gemm<CG, BV, kTerms, PAIR ? kChunk<PAIR> : 0, !PAIR, false, false>(logits, w, eg, tiles, sms, s);
        if (err != cudaSuccess) return cuda_fail(func, err, "launch the logits' gradient");
        // its contribution to dh
        w.tiles_n = ceil_div(p.width, BN);
        w.k = count;
        w.split_count = r.count + 1;
        w.n_fast = 1;
        es.add = i > 0;
        if (dh) err = launch_gemm<CG, BN, kTerms, PAIR ? kChunk<PAIR> : 0, !PAIR, false, true>(Maps{{gk[0], gk[1]}, {wm[0], wm[1]}}, w, es,
                                                                            ~uint64_t(0), sms, s);   // (all SMs)
        if (err != cudaSuccess) return cuda_fail(func, err, "launch the gradient of h");
        if (!dw) continue;
        // its rows of dW
        w = base;
        w.tiles_m = ceil_div(count, 256);
        w.tiles_n = ceil_div(p.width, BN);
        w.k = r.rows;
        w.k_count = r.count;
        w.n_fast = 1;
        T* out = static_cast<T*>(dw) + uint64_t(v0) * dw_stride;
        EpiWeight<T> ew{{}, out, dw_stride, r.scales, count, p.width, 0};
        ew.tma = mappable(out, static_cast<int64_t>(dw_stride), 16, count, 1, sizeof(T));
        if (ew.tma)
            if (int rc = make_map(func, &ew.to, out, p.width, count, 1, dw_stride, 0, 32, kOut)) return rc;
        err = launch_gemm<2, BN, kTerms, PAIR ? kChunk<PAIR> : 0, !PAIR, true, true>(Maps{{gm[0], gm[1]}, {hm[0], hm[1]}}, w, ew,
                                                                  uint64_t(w.tiles_m) * w.tiles_n, sms, s);
        if (err != cudaSuccess) return cuda_fail(func, err, "launch the gradient of W");
    }
    // (without dh only for the status)
    ScatterArgs sc{r.row,  r.target,  r.sum,      grad_loss, r.scales, grad_stride, r.count, r.count + 1,
                   r.rest, p.w,       dh_stride,  p.w_stride, r.ld_sum, p.tokens,   p.width, dh,
                   status, dw,        dw_stride,  p.vocab};
    const bool many = r.splits > 8;
    const uint64_t parts = dh ? uint64_t(p.tokens) * ceil_div(p.width, 128) : 0, blocks = many ? parts : ceil_div(parts, 8);
    const dim3 grid(static_cast<uint32_t>(blocks < 1 ? 1 : blocks < 4096 ? blocks : 4096));
    err = many ? launch_grid(k_ce_scatter<T, true>, grid, 256, 0, s, sc) : launch_grid(k_ce_scatter<T, false>, grid, 256, 0, s, sc);
    return err == cudaSuccess ? DSM_OK : cuda_fail(func, err, "launch the scatter of dh");
}

}  // namespace
}  // namespace ops
}  // namespace dsm

using namespace dsm;
using namespace dsm::ops;

extern "C" size_t dsm_linear_cross_entropy_workspace(const dsm_linear_ce* p, int grad) {
    const char* func = "dsm_linear_cross_entropy_workspace";
    if (check_args(func, p) != DSM_OK) return 0;
    dsm_linear_ce q = *p;
    if (!q.w) q.w = reinterpret_cast<const void*>(uintptr_t(2));  // unknown: as if it were not aligned
    return make_plan(q, grad != 0, nullptr).bytes;
}

extern "C" int dsm_linear_cross_entropy(const dsm_linear_ce* p, float* loss, float* lse, void* workspace,
                                        size_t workspace_bytes, dsm_stream_t stream) {
    const char* func = "dsm_linear_cross_entropy";
    if (int rc = check_args(func, p); rc != DSM_OK) return rc;
    if (int rc = check_vectors(func, *p, loss, lse, "loss and lse")) return rc;
    int dev = 0, sms = 0;
    if (int rc = device_of_call(func, &dev, &sms)) return rc;
    const Plan r = make_plan(*p, false, workspace);
    if (p->tokens && (!loss || !lse)) return fail(func, DSM_EINVAL, "NULL argument");
    if (int rc = check_call(func, p, r, workspace, workspace_bytes, dev)) return rc;
    if (p->tokens) {
        if (int rc = check_device(func, loss, "loss", dev)) return rc;
        if (int rc = check_device(func, lse, "lse", dev)) return rc;
    }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint32_t* status = static_cast<uint32_t*>(workspace);
    if (r.few) {
        FewArgs a = few_args(*p, r, status);
        a.loss = loss;
        a.lse = lse;
        const cudaError_t e = p->dtype == DSM_BF16 ? few<__nv_bfloat16>(a, r.few, false, sms, s) : few<float>(a, r.few, false, sms, s);
        return e == cudaSuccess ? DSM_OK : cuda_fail(func, e, "launch the loss of few tokens");
    }
    cudaError_t err = p->dtype == DSM_BF16 ? gather<__nv_bfloat16>(*p, r, nullptr, 0, false, status, s)
                                           : gather<float>(*p, r, nullptr, 0, false, status, s);
    if (err != cudaSuccess) return cuda_fail(func, err, "launch the gather");
    if (p->tokens == 0) return DSM_OK;
    const auto go = p->tokens > kPairRows ? (r.pair ? forward<true, 2> : forward<false, 2>)
                    : r.pair                ? forward<true, 1>
                    : r.tile_v == 128       ? forward<false, 1, 128>
                                            : forward<false, 1>;
    if (int rc = go(func, *p, r, status, sms, s)) return rc;
    JoinArgs j{r.count, r.row, r.target, r.token, r.partial, r.target_logit, loss, lse, p->tokens, r.groups, r.rows, status};
    const auto join = join_rows(p->tokens) == 8 ? k_ce_join<8> : k_ce_join<32>;
    err = launch_grid(join, dim3(ceil_div(p->tokens, join_rows(p->tokens))), 1024, 0, s, j);
    return err == cudaSuccess ? DSM_OK : cuda_fail(func, err, "launch the join");
}

extern "C" int dsm_linear_cross_entropy_grad(const dsm_linear_ce* p, const float* lse, const float* grad_loss,
                                             uint64_t grad_loss_stride, void* dh, uint64_t dh_stride, void* dw,
                                             uint64_t dw_stride, void* workspace, size_t workspace_bytes,
                                             dsm_stream_t stream) {
    const char* func = "dsm_linear_cross_entropy_grad";
    if (int rc = check_args(func, p); rc != DSM_OK) return rc;
    if (int rc = check_vectors(func, *p, lse, grad_loss, "lse and grad_loss")) return rc;
    int dev = 0, sms = 0;
    if (int rc = device_of_call(func, &dev, &sms)) return rc;
    const Plan r = make_plan(*p, true, workspace);
    if ((!dh && !dw) || (p->tokens && (!lse || !grad_loss))) return fail(func, DSM_EINVAL, "NULL argument");
    if (dh && dh_stride < p->width && p->tokens > 1) return fail(func, DSM_EINVAL, "dh_stride must be >= width");
    if (dw && dw_stride < p->width && p->vocab > 1) return fail(func, DSM_EINVAL, "dw_stride must be >= width");
    const uintptr_t esize = p->dtype == DSM_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(dh) % esize || reinterpret_cast<uintptr_t>(dw) % esize)
        return fail(func, DSM_EALIGN, "dh and dw must be aligned to their elements");
    if (int rc = check_call(func, p, r, workspace, workspace_bytes, dev)) return rc;
    if (dw)
        if (int rc = check_device(func, dw, "dw", dev)) return rc;
    if (p->tokens) {
        if (dh)
            if (int rc = check_device(func, dh, "dh", dev)) return rc;
        if (int rc = check_device(func, lse, "lse", dev)) return rc;
        if (int rc = check_device(func, grad_loss, "grad_loss", dev)) return rc;
    }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint32_t* status = static_cast<uint32_t*>(workspace);
    if (r.few) {
        FewArgs a = few_args(*p, r, status);
        a.lse_in = lse;
        a.grad_loss = grad_loss;
        a.grad_stride = grad_loss_stride;
        a.dh = dh;
        a.dw = dw;
        a.dh_stride = dh_stride;
        a.dw_stride = dw_stride;
        a.out_vec = reinterpret_cast<uintptr_t>(dw) % 16 == 0 && (p->vocab == 1 || dw_stride * esize % 16 == 0);
        const cudaError_t e = p->dtype == DSM_BF16 ? few<__nv_bfloat16>(a, r.few, true, sms, s) : few<float>(a, r.few, true, sms, s);
        return e == cudaSuccess ? DSM_OK : cuda_fail(func, e, "launch the gradient of few tokens");
    }
    cudaError_t err = p->dtype == DSM_BF16
                          ? gather<__nv_bfloat16>(*p, r, grad_loss, grad_loss_stride, dw != nullptr, status, s)
                          : gather<float>(*p, r, grad_loss, grad_loss_stride, dw != nullptr, status, s);
    if (err != cudaSuccess) return cuda_fail(func, err, "launch the gather");
    const auto go = p->tokens > kPairRows ? (r.pair ? backward<true, 2> : backward<false, 2>)
                    : r.pair                ? backward<true, 1>
                    : r.tile_v == 128       ? backward<false, 1, 128>
                                            : backward<false, 1>;
    return go(func, *p, r, lse, grad_loss, grad_loss_stride, dh, dh_stride, dw, dw_stride, status, sms, s);
}
