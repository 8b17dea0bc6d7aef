// dsm_orthogonalize: a weight matrix's update, orthogonalised by Newton-Schulz products.
//
// u = g, or with a momentum m <- mu m + g and u = m or g + mu m.  X_0 = u / max(|u|_F, eps); every step, with the
// smaller side m <= n first (a taller matrix is taken transposed, which only swaps the factors),
//   A = X X^T,  B = b A + c A A,  X <- a X + B X.
// The singular values go through the polynomial a s + b s^3 + c s^5; the singular vectors stay.
//
// Numbers.  The products run in f16 with f32 accumulators, every operand scaled by a power of two (kScale) so that it
// lies in f16's normal range: after the division by the norm all singular values are <= 1, and the polynomial's bound on
// them (checked on the host) keeps every entry below 2^16.  X is kept as a pair hi + lo of f16 (22 bits), of which the
// products take hi and a X takes both: what rounding hi loses is then not carried from step to step, where a would
// multiply it (3.4^5 over five steps, which on a matrix of low rank is all of the result); the last steps, in which it
// would not be multiplied by much any more, take hi alone.  B uses the same rounded A in
// both terms, so that A's rounding only moves the polynomial's argument.  A result in 32 bits takes pairs for A and B
// too and products of three terms.
#include <cmath>
#include <cstdlib>
#include <type_traits>

#include "orthogonalize.cuh"
#include "orthogonalize_small.cuh"

namespace dsm {
namespace ops {
namespace {

// The momentum's update and the partial sums of the squares of u, where g and the momentum lie along the columns: a warp
// takes 256 columns of a row, a thread 8 of them (VEC: consecutive ones, 16-byte accesses; else every 32nd).  u itself is
// not kept: k_orth_split computes it again from g and the momentum, for 6 bytes an element instead of 8.
// Bound by memory: 24 x 1024 x 4096 bf16 with momentum moves 10 bytes an element.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_orth_update(const __grid_constant__ UpdateArgs p) {
    __shared__ float2 sums[8];
    wait_previous();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = *p.barrier = 0;
    const uint64_t b = blockIdx.y;
    const T* g = static_cast<const T*>(p.g) + int64_t(b) * p.gs.batch;
    float* m = p.has_momentum ? p.momentum + int64_t(b) * p.ms.batch : nullptr;
    const uint32_t lane = threadIdx.x % 32, per_row = (p.cols + 255) / 256;
    float2 sum = make_float2(0.f, 0.f);
    for (uint32_t t = blockIdx.x * 8 + threadIdx.x / 32; t < p.rows * per_row; t += gridDim.x * 8) {
        const uint32_t r = t / per_row, c0 = t % per_row * 256;
        const T* gr = g + int64_t(r) * p.gs.row;
        float* mr = m ? m + int64_t(r) * p.ms.row : nullptr;
        __align__(16) float gv[8], mv[8] = {};
        if constexpr (VEC) {
            const uint32_t c = c0 + lane * 8;
            if (c >= p.cols) continue;
            __align__(16) T raw[8];
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
                reinterpret_cast<uint4*>(raw)[i] = *(reinterpret_cast<const uint4*>(gr + c) + i);
            if (mr) {
                *reinterpret_cast<float4*>(mv) = *reinterpret_cast<const float4*>(mr + c);
                *reinterpret_cast<float4*>(mv + 4) = *reinterpret_cast<const float4*>(mr + c + 4);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                gv[k] = to_float(raw[k]);
                if (mr) gv[k] = updated(p, gv[k], mv[k]);
                add_square(gv[k], sum);
            }
            if (mr) {
                *reinterpret_cast<float4*>(mr + c) = *reinterpret_cast<float4*>(mv);
                *reinterpret_cast<float4*>(mr + c + 4) = *reinterpret_cast<float4*>(mv + 4);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t c = c0 + lane + 32 * k;
                gv[k] = c < p.cols ? to_float(gr[c]) : 0.f;
                if (mr && c < p.cols) mv[k] = mr[c];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t c = c0 + lane + 32 * k;
                if (c >= p.cols) break;
                if (mr) {
                    gv[k] = updated(p, gv[k], mv[k]);
                    mr[c] = mv[k];
                }
                add_square(gv[k], sum);
            }
        }
    }
    sum = cta_sum(sum, sums);
    if (threadIdx.x == 0) p.partial[b * kUpdateBlocks + blockIdx.x] = sum;
}

// The same for any strides, with u kept in f32: tiles of 64 x 64 go through shared memory, so that each of g and m is walked along the
// dimension in which it is closer together.
template <typename T>
__global__ void __launch_bounds__(256) k_orth_update_strided(const __grid_constant__ UpdateArgs p) {
    __shared__ float tile[64][65];
    __shared__ float2 sums[8];
    wait_previous();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = *p.barrier = 0;
    const uint64_t b = blockIdx.y;
    const T* g = static_cast<const T*>(p.g) + int64_t(b) * p.gs.batch;
    float* m = p.has_momentum ? p.momentum + int64_t(b) * p.ms.batch : nullptr;
    float* u = p.u + b * p.rows * uint64_t(p.ld);
    const uint32_t tr = (p.rows + 63) / 64, tc = (p.cols + 63) / 64;
    const uint32_t lo = threadIdx.x % 64, hi = threadIdx.x / 64;
    const bool g_rows = llabs(p.gs.row) < llabs(p.gs.col), m_rows = llabs(p.ms.row) < llabs(p.ms.col);
    float2 sum = make_float2(0.f, 0.f);
    for (uint32_t t = blockIdx.x; t < tr * tc; t += gridDim.x) {
        const uint32_t r0 = t / tc * 64, c0 = t % tc * 64;
#pragma unroll 4
        for (uint32_t k = hi; k < 64; k += 4) {
            const uint32_t r = g_rows ? lo : k, c = g_rows ? k : lo;
            if (r0 + r < p.rows && c0 + c < p.cols)
                tile[r][c] = to_float(g[int64_t(r0 + r) * p.gs.row + int64_t(c0 + c) * p.gs.col]);
        }
        __syncthreads();
        if (m) {
#pragma unroll 4
            for (uint32_t k = hi; k < 64; k += 4) {
                const uint32_t r = m_rows ? lo : k, c = m_rows ? k : lo;
                if (r0 + r < p.rows && c0 + c < p.cols) {
                    float* at = m + int64_t(r0 + r) * p.ms.row + int64_t(c0 + c) * p.ms.col;
                    float mv = *at;
                    tile[r][c] = updated(p, tile[r][c], mv);
                    *at = mv;
                }
            }
            __syncthreads();
        }
        for (uint32_t k = hi; k < 64; k += 4)
            if (r0 + k < p.rows && c0 + lo < p.cols) {
                const float v = tile[k][lo];
                add_square(v, sum);
                u[uint64_t(r0 + k) * p.ld + c0 + lo] = v;
            }
        __syncthreads();
    }
    sum = cta_sum(sum, sums);
    if (threadIdx.x == 0) p.partial[b * kUpdateBlocks + blockIdx.x] = sum;
}

struct SplitArgs {
    UpdateArgs in;            // DIRECT: g and the updated momentum
    __half *hi, *lo;          // lo: null where it is not needed
    uint32_t blocks;          // partial sums per matrix
    float eps;
    // steps = 0: the result is scale * u / max(|u|, eps), written here
    void* out;
    Strides os;
    float scale;
    int out_bf16;
};

// X_0 from u, as hi + lo: a warp takes 256 columns of a row, a thread 8 of them.  DIRECT: u from g and the momentum, which
// lie along the columns (VEC: on 16-byte boundaries); else the f32 u.
template <typename T, bool DIRECT, bool VEC>
__global__ void __launch_bounds__(256) k_orth_split(const __grid_constant__ SplitArgs p) {
    __shared__ float2 sums[8];
    wait_previous();
    const UpdateArgs& in = p.in;
    const uint64_t b = gridDim.y - 1 - blockIdx.y;   // the other way round: the last matrices' data may still be in L2
    float2 v = make_float2(0.f, 0.f);
    if (threadIdx.x < p.blocks) v = in.partial[b * kUpdateBlocks + threadIdx.x];
    v = cta_sum(v, sums);
    const Unit unit = to_unit(v, p.eps);
    const uint32_t lane = threadIdx.x % 32, per_row = (in.cols + 255) / 256;
    for (uint32_t t = blockIdx.x * 8 + threadIdx.x / 32; t < in.rows * per_row; t += gridDim.x * 8) {
        const uint32_t r = t / per_row, c = t % per_row * 256 + lane * 8;
        if (c >= in.cols) continue;
        __align__(16) float x[8] = {}, m[8] = {};
        if constexpr (DIRECT) {
            const T* g = static_cast<const T*>(in.g) + int64_t(b) * in.gs.batch + int64_t(r) * in.gs.row + c;
            const float* mr = in.momentum + int64_t(b) * in.ms.batch + int64_t(r) * in.ms.row + c;
            if constexpr (VEC) {
                __align__(16) T raw[8];
#pragma unroll
                for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
                    reinterpret_cast<uint4*>(raw)[i] = *(reinterpret_cast<const uint4*>(g) + i);
                if (in.has_momentum) {
                    *reinterpret_cast<float4*>(m) = *reinterpret_cast<const float4*>(mr);
                    *reinterpret_cast<float4*>(m + 4) = *reinterpret_cast<const float4*>(mr + 4);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = to_float(raw[k]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (c + k >= in.cols) break;
                    x[k] = to_float(g[k]);
                    if (in.has_momentum) m[k] = mr[k];
                }
            }
            if (in.has_momentum)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = in.nesterov ? fmaf(in.mu, m[k], x[k]) : m[k];
        } else {
            const float* u = in.u + (b * in.rows + r) * uint64_t(in.ld) + c;   // (what lies behind the last column is not used)
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(u);
            *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(u + 4);
        }
        if (p.out) {
            for (int k = 0; k < 8; ++k) {
                if (c + k >= in.cols) break;
                const float y = unit(x[k]) * p.scale;
                const int64_t at = int64_t(b) * p.os.batch + int64_t(r) * p.os.row + int64_t(c + k) * p.os.col;
                if (p.out_bf16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(y);
                else static_cast<float*>(p.out)[at] = y;
            }
            continue;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = unit(x[k]) * kScale;
        const uint64_t at = (b * in.rows + r) * uint64_t(in.ld) + c;
        const uint4 hi = pack8<__half>(x);
        *reinterpret_cast<uint4*>(p.hi + at) = hi;
        if (p.lo) *reinterpret_cast<uint4*>(p.lo + at) = rest8<__half>(x, hi);
    }
}

// The epilogues.  What they read and write of the matrices X, A and B goes through the warp's buffer by TMA, 64 columns
// at a time: hi in the buffer's first 4 KB, lo in the second.

// Starts the load of the pair (x, y) of a matrix.
template <bool PAIR>
__device__ __forceinline__ void load_pair(const CUtensorMap (&maps)[2], uint32_t x, uint32_t y, uint32_t z, const WarpBuffer& buf) {
    if (buf.lane == 0) {
        tma_store_wait_read();
        mbar_expect(buf.bar, PAIR ? 8192 : 4096);
        tma_fetch(buf.addr, &maps[0], buf.bar, x, y, z);
        if constexpr (PAIR) tma_fetch(buf.addr + 4096, &maps[1], buf.bar, x, y, z);
    }
    __syncwarp();
}

// Where a symmetric m x m matrix is stored: its hi and lo, and both for mirror images.
template <bool PAIR>
struct Symmetric {
    CUtensorMap to[2], mirror[2];
    uint32_t m, square;          // square: the side of the schedule's squares

    // Columns [x, x + 64) of the rows from y, as f16 hi and (PAIR) lo, and the same values mirrored where no tile of this
    // product covers the mirror image.
    __device__ __forceinline__ void store(const float (&v)[64], uint32_t x, uint32_t y, const Tile& t, const WarpBuffer& buf) const {
        const bool twice = t.n0 / square > t.m0 / square;
        uint4 h[8], l[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            h[j] = pack8<__half>(v + 8 * j);
            sts128(buf.at(j), h[j]);
            if constexpr (PAIR) {
                l[j] = rest8<__half>(v + 8 * j, h[j]);
                sts128(buf.at(j) + 4096, l[j]);
            }
        }
        // the mirror image, 64 rows of 32 columns: a row is a column of the warp's, 64 consecutive bytes
        auto turn = [&](uint32_t at, const uint4 (&from)[8]) {
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                const uint4& e = from[k / 4];
                const uint32_t two = k % 4 == 0 ? e.x : k % 4 == 1 ? e.y : k % 4 == 2 ? e.z : e.w;
                sts16(at + 2 * k * 64 + buf.lane * 2, static_cast<uint16_t>(two));
                sts16(at + (2 * k + 1) * 64 + buf.lane * 2, static_cast<uint16_t>(two >> 16));
            }
        };
        if (twice && !PAIR) turn(buf.addr + 4096, h);
        if (buf.written()) {
            tma_store(&to[0], buf.addr, x, y, t.batch);
            if constexpr (PAIR) tma_store(&to[1], buf.addr + 4096, x, y, t.batch);
            else if (twice) tma_store(&mirror[0], buf.addr + 4096, y, x, t.batch);
            tma_store_commit();
        }
        if (PAIR && twice) {
            buf.reuse();
            turn(buf.addr, h);
            turn(buf.addr + 4096, l);
            if (buf.written()) {
                tma_store(&mirror[0], buf.addr, y, x, t.batch);
                tma_store(&mirror[1], buf.addr + 4096, y, x, t.batch);
                tma_store_commit();
            }
        }
    }
};

// A = X X^T (or X^T X).
template <bool PAIR>
struct EpiGram {
    Symmetric<PAIR> out;
    __device__ __forceinline__ void before(const Tile&, uint32_t, uint32_t, const WarpBuffer&) const {}
    template <int COLUMNS, class Columns>
    __device__ __forceinline__ bool tile(const Tile& t, uint32_t row, uint32_t col, const Columns& acc, bool, WarpBuffer& buf) const {
#pragma unroll
        for (int c = 0; c < COLUMNS; c += 64) {
            __align__(16) float v[64];
            acc.load(c, *reinterpret_cast<float(*)[32]>(v));
            acc.load(c + 32, *reinterpret_cast<float(*)[32]>(v + 32));
            if (c + 64 == COLUMNS) acc.done();
            if (row >= out.m || col + c >= out.m) continue;
#pragma unroll
            for (int k = 0; k < 64; ++k) v[k] *= 1.f / kScale;
            buf.reuse();
            out.store(v, col + c, row, t, buf);
        }
        return true;
    }
};

// B = b A + c A A.
template <bool PAIR>
struct EpiSquare {
    Symmetric<PAIR> out;
    CUtensorMap from[2];         // A
    struct Step {
        const EpiSquare& e;
        float b, c;
        __device__ __forceinline__ void before(const Tile& t, uint32_t row, uint32_t col, const WarpBuffer& buf) const {
            if (row < e.out.m && col < e.out.m) load_pair<PAIR>(e.from, col, row, t.batch, buf);
        }
        template <int COLUMNS, class Columns>
        __device__ __forceinline__ bool tile(const Tile& t, uint32_t row, uint32_t col, const Columns& acc, bool, WarpBuffer& buf) const {
            return e.template store<COLUMNS>(t, row, col, acc, b, c, buf);
        }
    };
    template <int COLUMNS, class Columns>
    __device__ __forceinline__ bool store(const Tile& t, uint32_t row, uint32_t col, const Columns& acc, float b, float c,
                                          WarpBuffer& buf) const {
#pragma unroll
        for (int x = 0; x < COLUMNS; x += 64) {
            __align__(16) float v[64];
            acc.load(x, *reinterpret_cast<float(*)[32]>(v));
            acc.load(x + 32, *reinterpret_cast<float(*)[32]>(v + 32));
            if (x + 64 == COLUMNS) acc.done();
            if (row >= out.m || col + x >= out.m) continue;
            if (x) load_pair<PAIR>(from, col + x, row, t.batch, buf);
            if (!buf.wait_load()) return false;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4 h = lds128(buf.at(j)), l = PAIR ? lds128(buf.at(j) + 4096) : uint4{};
                float a[8];
                unpack8<__half, PAIR>(h, l, a);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[8 * j + k] = fmaf(c * (1.f / kScale), v[8 * j + k], b * a[k]);
            }
            out.store(v, col + x, row, t, buf);
        }
        return true;
    }
};

// X <- a X + B X (or X B); the last step's goes out instead, times scale: by TMA (but for the ragged end of rows), or by
// plain stores with neighbouring threads on neighbouring columns or rows.
enum class Out { none, tma, columns, rows };
template <typename T>
struct EpiApply {
    static constexpr uint32_t kBuffer = 8192;
    static constexpr bool kPair = sizeof(T) == 4;
    CUtensorMap from[2], to[2];
    uint32_t rows, cols;
    T* out;
    Strides os;
    float scale;                 // includes 1 / kScale
    struct Step {
        const EpiApply& e;
        const CUtensorMap& map;  // of out
        float a;
        Out mode;
        bool lo_in, lo_out;      // whether X, and the next X, are pairs
        // Without lo the warp's 128 columns fit into its buffer: both halves are loaded at once.
        __device__ __forceinline__ bool whole() const { return !kPair && !lo_in && !lo_out; }
        __device__ __forceinline__ void before(const Tile& t, uint32_t row, uint32_t col, const WarpBuffer& buf) const {
            if (row >= e.rows || col >= e.cols) return;
            if (!whole()) return load(t, row, col, buf);
            if (buf.lane == 0) {
                const bool two = buf.columns > 64 && col + 64 < e.cols;
                tma_store_wait_read();
                mbar_expect(buf.bar, two ? 8192 : 4096);
                tma_fetch(buf.addr, &e.from[0], buf.bar, col, row, t.batch);
                if (two) tma_fetch(buf.addr + 4096, &e.from[0], buf.bar, col + 64, row, t.batch);
            }
            __syncwarp();
        }
        __device__ __forceinline__ void load(const Tile& t, uint32_t row, uint32_t col, const WarpBuffer& buf) const {
            if (kPair || lo_in) load_pair<true>(e.from, col, row, t.batch, buf);
            else load_pair<false>(e.from, col, row, t.batch, buf);
        }
        template <int COLUMNS, class Columns>
        __device__ __forceinline__ bool tile(const Tile& t, uint32_t row, uint32_t col, const Columns& acc, bool, WarpBuffer& buf) const {
            return e.template store<COLUMNS>(t, row, col, acc, *this, buf);
        }
    };
    template <int COLUMNS, class Columns>
    __device__ __forceinline__ bool store(const Tile& t, uint32_t row, uint32_t col, const Columns& acc, const Step& step,
                                          WarpBuffer& buf) const {
        const Out mode = step.mode;
        const bool lo_in = kPair || step.lo_in, lo_out = kPair || step.lo_out;
#pragma unroll
        for (int x = 0; x < COLUMNS; x += 64) {
            __align__(16) float v[64];
            acc.load(x, *reinterpret_cast<float(*)[32]>(v));
            acc.load(x + 32, *reinterpret_cast<float(*)[32]>(v + 32));
            if (x + 64 == COLUMNS) acc.done();
            if (row >= rows || col + x >= cols) continue;
            const bool whole = step.whole();
            const uint32_t half = whole ? x / 64 * 4096 : 0;   // of the buffer
            if (x && !whole) step.load(t, row, col + x, buf);
            if (!(x && whole) && !buf.wait_load()) return false;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4 h = lds128(buf.at(j) + half), l = lo_in ? lds128(buf.at(j) + 4096) : uint4{};
                float was[8];
                unpack8<__half, true>(h, l, was);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[8 * j + k] = fmaf(step.a, was[k], v[8 * j + k] * (1.f / kScale));
            }
            if (mode == Out::none) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint4 h = pack8<__half>(v + 8 * j);
                    sts128(buf.at(j) + half, h);
                    if (lo_out) sts128(buf.at(j) + 4096, rest8<__half>(v + 8 * j, h));
                }
                if (buf.written()) {
                    tma_store(&to[0], buf.addr + half, col + x, row, t.batch);
                    if (lo_out) tma_store(&to[1], buf.addr + 4096, col + x, row, t.batch);
                    tma_store_commit();
                }
                continue;
            }
            T* o = out + int64_t(t.batch) * os.batch;
            if (mode == Out::rows) {
                if (row + buf.lane < rows) {
                    o += int64_t(row + buf.lane) * os.row;
#pragma unroll
                    for (int k = 0; k < 64; ++k)
                        if (col + x + k < cols) o[int64_t(col + x + k) * os.col] = round_to<T>(v[k] * scale);
                }
                __syncwarp();
                continue;
            }
            __syncwarp();  // all threads have read their rows; 4-byte results fill both halves of the buffer
            constexpr int kPer = 16 / sizeof(T);
#pragma unroll
            for (int k = 0; k < 64; ++k) v[k] *= scale;
#pragma unroll
            for (int j = 0; j < 64 / kPer; ++j) {
                uint4 r;
                if constexpr (sizeof(T) == 4) r = *reinterpret_cast<const uint4*>(v + 4 * j);
                else r = pack8<T>(v + 8 * j);
                sts128(buf.at(j % 8) + j / 8 * 4096 + half, r);
            }
            if (mode == Out::tma && ends_whole<T>(col + x + 64, cols)) {
                if (buf.written()) {
                    tma_store(&step.map, buf.addr + half, col + x, row, t.batch);
                    if constexpr (sizeof(T) == 4) tma_store(&step.map, buf.addr + 4096, col + x + 32, row, t.batch);
                    tma_store_commit();
                }
                continue;
            }
            __syncwarp();
            constexpr int kBox = 128 / sizeof(T);
#pragma unroll
            for (int c = 0; c < 64; c += kBox)
                if (col + x + c < cols)
                    store_box(buf.addr + c / kBox * 4096 + half, buf.lane, o + int64_t(row) * os.row + int64_t(col + x + c) * os.col,
                              os.row, os.col, rows - row, cols - (col + x + c));
            fence_async_smem();  // the buffer's next writer is TMA
            __syncwarp();
        }
        return true;
    }
};

constexpr const char* kFunc = "dsm_orthogonalize";
constexpr uint64_t kMaxSide = 1u << 20;

struct Plan {
    // The matrices are taken with their columns along memory: transposed if most of g, out and the momentum lie so.
    // A transposed matrix has the transposed result.
    bool flip;
    uint32_t rows, cols, m;   // m: the smaller side
    uint32_t ldx, lda;
    uint64_t x_plane, a_plane;
    __half *x[2][2], *a[2], *b[2];   // x: [ping][hi, lo]
    float* u;
    float2* partial;
    uint32_t* barrier;
    uint64_t bytes;
    uint32_t pairs;           // as StepsArgs::pairs
    Strides oriented(const int64_t (&v)[3]) const { return Strides{v[0], flip ? v[2] : v[1], flip ? v[1] : v[2]}; }
};

// Where everything lies in the workspace.  Its size does not depend on the strides.
Plan make_plan(const dsm_orthogonalize_args& p, void* workspace) {
    auto down = [](const int64_t (&v)[3]) { return llabs(v[1]) < llabs(v[2]) ? 1 : -1; };
    Plan r{};
    r.flip = down(p.g_stride) + down(p.out_stride) + (p.momentum ? 2 * down(p.momentum_stride) : 0) > 0;
    r.rows = static_cast<uint32_t>(r.flip ? p.cols : p.rows);
    r.cols = static_cast<uint32_t>(r.flip ? p.rows : p.cols);
    r.m = r.rows < r.cols ? r.rows : r.cols;
    r.ldx = static_cast<uint32_t>(round_up(r.cols, 8));
    r.lda = static_cast<uint32_t>(round_up(r.m, 8));
    r.x_plane = uint64_t(r.rows) * r.ldx;
    r.a_plane = uint64_t(r.m) * r.lda;
    const uint64_t most = uint64_t(round_up(r.rows, 8)) * round_up(r.cols, 8);   // of both orientations
    Carver c(workspace);
    for (int i = 0; i < 2; ++i) r.x[0][i] = c.take<__half>(p.count * most);
    // u is read by the split, which writes the first pair: it shares the second pair's memory
    __half* second = c.take<__half>(2 * round_up(p.count * most, 128));
    r.x[1][0] = second;
    r.x[1][1] = second ? second + round_up(p.count * most, 128) : nullptr;
    r.u = reinterpret_cast<float*>(second);
    const int parts = p.dtype == DSM_F32 ? 2 : 1;
    for (int i = 0; i < parts; ++i) {
        r.a[i] = c.take<__half>(p.count * r.a_plane);
        r.b[i] = c.take<__half>(p.count * r.a_plane);
    }
    r.partial = c.take<float2>(uint64_t(p.count) * kUpdateBlocks);
    r.barrier = c.take<uint32_t>(1);
    r.bytes = c.used;
    return r;
}

// The most that a step makes of singular values x in [0, top]: of p(x) = (a + q(x^2)) x with q(l) = b l + c l^2, of q, and
// of p's derivative a + 3 b l + 5 c l^2, at the ends and where their derivatives (in l) are zero.
struct Bounds {
    double value, q, slope;
};
Bounds bounds_of(const float* coefficients, double top) {
    const double a = coefficients[0], b = coefficients[1], c = coefficients[2], end = top * top;
    Bounds r{0, 0, 0};
    auto at = [&](double l) {
        if (!(l >= 0 && l <= end)) return;   // (no such point: NaN or infinite)
        r.value = std::fmax(r.value, std::fabs((a + b * l + c * l * l) * std::sqrt(l)));
        r.q = std::fmax(r.q, std::fabs(b * l + c * l * l));
        r.slope = std::fmax(r.slope, std::fabs(a + 3 * b * l + 5 * c * l * l));
    };
    at(0);
    at(end);
    const double root = std::sqrt(9 * b * b - 20 * a * c);
    at((-3 * b + root) / (10 * c));
    at((-3 * b - root) / (10 * c));
    at(-a / (3 * b));                        // c = 0
    at(-b / (2 * c));
    at(-3 * b / (10 * c));
    return r;
}

// X of step k (from 0) is kept as a pair if what is lost of it may be multiplied by more than 16 in the steps from k on:
// 16 * 2^-12 / sqrt(12) is 1e-3 of the norm of a matrix of rank 1.  (The first three of five steps with a = 3.4445.)
uint32_t count_pairs(const dsm_orthogonalize_args& p) {
    double gain[DSM_ORTHOGONALIZE_MAX_STEPS], top = 1, all = 1;
    for (uint32_t k = 0; k < p.steps; ++k) {
        const Bounds b = bounds_of(p.coefficients + 3 * k, top);
        gain[k] = b.slope;
        top = b.value;
    }
    uint32_t k = p.steps;
    while (k > 0 && (all *= gain[k - 1]) <= 16) --k;
    return k;
}

bool finite(float v) { return v - v == 0.f; }

// The checks of the arguments that need no device.
int check_args(const char* func, const dsm_orthogonalize_args* p) {
    if (!p) return fail(func, DSM_EINVAL, "NULL argument");
    if (p->dtype != DSM_F32 && p->dtype != DSM_BF16) return fail(func, DSM_EINVAL, "dtype %d unknown", p->dtype);
    if (p->reserved) return fail(func, DSM_EINVAL, "reserved must be 0");
    if (p->count > 65535) return fail(func, DSM_ERANGE, "count must be at most 65535");
    if (p->rows > kMaxSide || p->cols > kMaxSide) return fail(func, DSM_ERANGE, "rows and cols must be at most 2^20");
    if (p->steps > DSM_ORTHOGONALIZE_MAX_STEPS)
        return fail(func, DSM_ERANGE, "steps must be at most DSM_ORTHOGONALIZE_MAX_STEPS (%d)", DSM_ORTHOGONALIZE_MAX_STEPS);
    if (p->steps && !p->coefficients) return fail(func, DSM_EINVAL, "coefficients must not be NULL");
    if (!(p->eps > 0.f && finite(p->eps))) return fail(func, DSM_EINVAL, "eps must be finite and > 0");
    if (!finite(p->scale)) return fail(func, DSM_EINVAL, "scale must be finite");
    if (!finite(p->mu) || p->mu < 0.f || p->mu >= 1.f) return fail(func, DSM_EINVAL, "mu must lie in [0, 1)");
    // The singular values' bound through the steps: X, A = X X^T and b A + c A A have to stay in f16's range.
    double top = 1.0;
    for (uint32_t s = 0; s < p->steps; ++s) {
        const float* at = p->coefficients + 3 * s;
        if (!finite(at[0]) || !finite(at[1]) || !finite(at[2]))
            return fail(func, DSM_EINVAL, "step %u's coefficients are not finite", s);
        const Bounds b = bounds_of(at, top * 1.01);   // 1 % for rounding
        if (!(b.value < 3.5 && b.q < 15.0))
            return fail(func, DSM_EINVAL, "step %u's coefficients let the singular values grow beyond 3.5", s);
        top = b.value;
    }
    return DSM_OK;
}

// All steps as one cooperative launch: the products of a step one after another, all CTAs of the grid between them.
// (A kernel per product starts, sets itself up and ends fifteen times: 768 x 768 in 119 us.)
template <bool PAIR>
struct StepsArgs {
    Maps gram[2], square, apply[2];              // operands, by the X they read
    EpiGram<PAIR> to_gram;
    EpiSquare<PAIR> to_square;
    EpiApply<std::conditional_t<PAIR, float, __nv_bfloat16>> to_apply[2];
    Schedule half_n, half_m, all;                // of the three products
    uint32_t* barrier;
    uint32_t gave_up;                            // injected_timeout()
    uint32_t steps, pairs;                       // X of the first `pairs` steps are pairs (of all, for a result in 32 bits)
    Out last;                                    // where the last step's result goes
    CUtensorMap out;
    float coefficients[3 * DSM_ORTHOGONALIZE_MAX_STEPS];
};

template <class S, bool PAIR, bool TALL>
__global__ void __launch_bounds__(S::kThreads, 1) k_orth_steps(const __grid_constant__ StepsArgs<PAIR> a) {
    extern __shared__ uint8_t raw[];
    Pipe<S> p;
    p.open(raw);
    p.ok = !a.gave_up;
    wait_previous();
    using Sched = Scheduler<S>;
    const Sched half_n(a.half_n), half_m(a.half_m), all(a.all);
    GridBarrier grid{a.barrier};
    // One product; every role for itself.  `ready`: B is not what the last product has written.
    auto product = [&](auto a_mn, auto b_mn, bool ready, const Maps& maps, const Sched& sched, const auto& epi) {
        constexpr bool A_MN = decltype(a_mn)::value, B_MN = decltype(b_mn)::value;
        if (!p.ok) return;
        // A's producer waits for the grid and passes it on: one warp of the CTA asks, not ten.
        auto wait = [&] {
            p.ok = !grid.phase || warp_wait(p.go(), (grid.phase - 1) & 1);
            asm volatile("fence.proxy.async;" ::: "memory");
            return p.ok;
        };
        if (p.producer_a()) {
            if (grid.phase) {
                if (!(p.ok = __all_sync(0xffffffffu, grid.wait(gridDim.x)))) return;
                if (elect_one()) mbar_arrive(p.go());
                __syncwarp();
            }
            if (elect_one()) produce<false, A_MN>(p, maps.a, sched);
            p.meet();
        } else if (p.producer_b()) {
            if (!ready && !wait()) return;
            if (elect_one()) produce<true, B_MN>(p, maps.b, sched);
            p.meet();
            if (ready && (!p.ok || !wait())) return;   // (every phase of the barrier has to be seen: it has two states)
        } else if (p.multiplier()) {
            if (elect_one()) multiply<A_MN, B_MN>(p, sched);
            p.meet();
        } else if (p.finisher()) {
            if (!wait()) return;
            finish(p, sched, epi);
            if (p.ok) grid.arrive(p.done_warps(), S::kEpiWarps);
        }
        ++grid.phase;
    };
    using Tall = std::bool_constant<TALL>;
    using Wide = std::bool_constant<!TALL>;
    for (uint32_t k = 0; k < a.steps; ++k) {
        const uint32_t now = k & 1;
        product(Tall{}, Tall{}, false, a.gram[now], half_n, a.to_gram);
        product(std::false_type{}, std::false_type{}, false, a.square, half_m,
                typename EpiSquare<PAIR>::Step{a.to_square, a.coefficients[3 * k + 1], a.coefficients[3 * k + 2]});
        using Apply = std::remove_cv_t<std::remove_reference_t<decltype(a.to_apply[0])>>;
        product(std::false_type{}, Wide{}, !TALL, a.apply[now], all,
                typename Apply::Step{a.to_apply[now], a.out, a.coefficients[3 * k], k + 1 == a.steps ? a.last : Out::none,
                                     k < a.pairs, k + 1 < a.pairs});
    }
    p.close(a.all.status);
    // A CTA that gave up has left tiles unwritten, which no other writes.
    if (__syncthreads_or(!p.ok)) {
        const auto& e = a.to_apply[0];
        fill_nan(e.out, a.all.batches, e.rows, e.cols, e.os.batch, e.os.row, e.os.col, threadIdx.x, S::kThreads);
    }
}

template <int CG, int BN, bool PAIR, bool TALL>
int steps(const dsm_orthogonalize_args& p, const Plan& r, uint32_t* status, int dev, cudaStream_t s) {
    using T = std::conditional_t<PAIR, float, __nv_bfloat16>;
    using S = Shape<CG, BN, PAIR ? 3 : 1, PAIR ? 128 : 0, false, EpiApply<T>::kBuffer>;
    constexpr uint32_t kBM = 128 * CG, kSquare = kBM > BN ? kBM : BN, kRowsB = BN / CG;
    StepsArgs<PAIR> a{};
    a.to_gram.out.m = a.to_square.out.m = r.m;
    a.to_gram.out.square = a.to_square.out.square = kSquare;
    const Strides os = r.oriented(p.out_stride);
    for (int i = 0; i < 2; ++i) {
        const __half *ga = r.a[PAIR ? i : 0], *gb = r.b[PAIR ? i : 0];
        auto square = [&](CUtensorMap* map, const __half* of, uint32_t rows) {
            return make_map(kFunc, map, of, r.m, r.m, p.count, r.lda, r.a_plane, rows, Elem::f16);
        };
        for (int ping = 0; ping < 2; ++ping) {
            auto x = [&](CUtensorMap* map, uint32_t rows) {
                return make_map(kFunc, map, r.x[ping][i], r.cols, r.rows, p.count, r.ldx, r.x_plane, rows, Elem::f16);
            };
            // wide: X X^T over the columns, B X;  tall: X^T X over the rows, X B
            if (int rc = x(&a.gram[ping].a[i], TALL ? 64 : 128)) return rc;
            if (int rc = x(&a.gram[ping].b[i], TALL ? 64 : kRowsB)) return rc;
            if (int rc = TALL ? x(&a.apply[ping].a[i], 128) : square(&a.apply[ping].a[i], gb, 128)) return rc;
            if (int rc = TALL ? square(&a.apply[ping].b[i], gb, kRowsB) : x(&a.apply[ping].b[i], 64)) return rc;
            if (int rc = x(&a.to_apply[ping].from[i], 32)) return rc;
            a.to_apply[ping ^ 1].to[i] = a.to_apply[ping].from[i];
        }
        if (int rc = square(&a.square.a[i], ga, 128)) return rc;
        if (int rc = square(&a.square.b[i], ga, kRowsB)) return rc;
        if (int rc = square(&a.to_gram.out.to[i], ga, 32)) return rc;
        if (int rc = square(&a.to_square.out.to[i], gb, 32)) return rc;
        a.to_square.from[i] = a.to_gram.out.to[i];
        auto mirror = [&](CUtensorMap* map, const __half* of) {
            return make_plain_map(kFunc, map, of, r.m, r.m, p.count, r.lda, r.a_plane, 64, Elem::f16);
        };
        if (int rc = mirror(&a.to_gram.out.mirror[i], ga)) return rc;
        if (int rc = mirror(&a.to_square.out.mirror[i], gb)) return rc;
    }
    for (EpiApply<T>& e : a.to_apply) {
        e.rows = r.rows;
        e.cols = r.cols;
        e.out = static_cast<T*>(p.out);
        e.os = os;
        e.scale = p.scale / kScale;
    }
    const bool tma = os.col == 1 && mappable(p.out, os.row, os.batch, r.rows, p.count, sizeof(T));
    a.last = tma ? Out::tma : os.row == 1 ? Out::rows : Out::columns;
    if (tma)
        if (int rc = make_map(kFunc, &a.out, p.out, r.cols, r.rows, p.count, os.row, os.batch, 32, PAIR ? Elem::f32 : Elem::bf16))
            return rc;
    Schedule w{};
    w.batches = p.count;
    w.splits = 1;
    w.n_fast = 1;
    w.status = status;
    a.half_n = a.half_m = a.all = w;
    a.half_n.symmetric = a.half_m.symmetric = 1;
    a.half_n.tiles_m = a.half_n.tiles_n = a.half_m.tiles_m = a.half_m.tiles_n = ceil_div(r.m, kSquare);
    a.half_n.k = TALL ? r.rows : r.cols;
    a.half_m.k = a.all.k = r.m;
    a.all.tiles_m = ceil_div(r.rows, kBM);
    a.all.tiles_n = ceil_div(r.cols, BN);
    a.barrier = r.barrier;
    a.gave_up = injected_timeout();
    a.steps = p.steps;
    a.pairs = r.pairs;
    for (uint32_t i = 0; i < 3 * p.steps; ++i) a.coefficients[i] = p.coefficients[i];
    const uint64_t q = a.half_n.tiles_m, half = q * (q + 1) / 2 * (kSquare / kBM) * (kSquare / BN) * p.count;
    const uint64_t all = uint64_t(a.all.tiles_m) * a.all.tiles_n * p.count, most = half > all ? half : all;
    static std::atomic<int> known[64];
    const cudaError_t err = launch_together(k_orth_steps<S, PAIR, TALL>, most, CG, S::kThreads, S::kSmem, dev, known, s, a);
    return err == cudaSuccess ? DSM_OK : cuda_fail(kFunc, err, "launch the steps");
}

template <int CG, int BN, bool PAIR>
int steps(const dsm_orthogonalize_args& p, const Plan& r, uint32_t* status, int dev, cudaStream_t s) {
    return r.rows > r.cols ? steps<CG, BN, PAIR, true>(p, r, status, dev, s) : steps<CG, BN, PAIR, false>(p, r, status, dev, s);
}

// Clocks of one step's products with tiles of 128 cg x bn: rounds of the SMs (or pairs) over the tiles, times a tile's
// blocks of k and what a tile costs besides.  A block takes what its matrix instructions take at 8192 products a clock and
// SM, or the loads of a stage at 70 bytes a clock and SM, or the 170 clocks of issuing it.
uint64_t step_clocks(const Plan& r, uint32_t count, int sms, uint32_t cg, uint32_t bn, uint32_t terms) {
    const uint32_t bm = 128 * cg, square = bn > bm ? bn : bm, q = ceil_div(r.m, square), n = r.rows > r.cols ? r.rows : r.cols;
    const uint32_t units = sms / cg;
    const uint64_t half = uint64_t(q) * (q + 1) / 2 * (square / bm) * (square / bn) * count;
    const uint64_t all = uint64_t(ceil_div(r.rows, bm)) * ceil_div(r.cols, bn) * count;
    const uint32_t mma = 2 * bn * terms, load = (128 + bn / cg) * 128 * (terms == 3 ? 2 : 1) / 70;
    const uint32_t block = mma > load ? (mma > 170 ? mma : 170) : (load > 170 ? load : 170);
    const uint64_t fixed = 3000 + 10 * bn, kn = ceil_div(n, kBlockK), km = ceil_div(r.m, kBlockK);
    return ceil_div(half, units) * ((kn + km) * block + 2 * fixed) + ceil_div(all, units) * (km * block + fixed);
}

// The first two kernels: the momentum's update with the norms, and X_0 (or the result of no steps).
template <typename T>
cudaError_t launch_start(const dsm_orthogonalize_args& p, const Plan& r, uint32_t* status, cudaStream_t s) {
    SplitArgs sp{};
    UpdateArgs& up = sp.in;
    up.g = p.g;
    up.momentum = p.momentum;
    up.has_momentum = p.momentum != nullptr;
    up.u = r.u;
    up.partial = r.partial;
    up.status = status;
    up.barrier = r.barrier;
    up.gs = r.oriented(p.g_stride);
    up.ms = r.oriented(p.momentum_stride);
    up.rows = r.rows;
    up.cols = r.cols;
    up.ld = r.ldx;
    up.mu = p.mu;
    up.nesterov = p.nesterov;
    const bool along = up.gs.col == 1 && (!p.momentum || up.ms.col == 1);
    auto aligned = [&](const void* base, const Strides& v, int esize) {
        return reinterpret_cast<uintptr_t>(base) % 16 == 0 && v.row * esize % 16 == 0 && v.batch * esize % 16 == 0;
    };
    const bool vec = along && r.cols % 8 == 0 && aligned(p.g, up.gs, sizeof(T)) && (!p.momentum || aligned(p.momentum, up.ms, 4));
    const uint64_t rows = ceil_div(uint64_t(r.rows) * ceil_div(r.cols, 256), 8), tiles = uint64_t(ceil_div(r.rows, 64)) * ceil_div(r.cols, 64);
    const uint64_t parts = along ? rows : tiles;
    sp.blocks = parts < kUpdateBlocks ? static_cast<uint32_t>(parts) : kUpdateBlocks;
    dim3 grid(sp.blocks, p.count);
    cudaError_t err = vec     ? launch_grid(k_orth_update<T, true>, grid, 256, 0, s, up)
                      : along ? launch_grid(k_orth_update<T, false>, grid, 256, 0, s, up)
                              : launch_grid(k_orth_update_strided<T>, grid, 256, 0, s, up);
    if (err != cudaSuccess) return err;
    sp.hi = r.x[0][0];
    sp.lo = r.pairs ? r.x[0][1] : nullptr;
    sp.eps = p.eps;
    sp.out = p.steps ? nullptr : p.out;
    sp.os = r.oriented(p.out_stride);
    sp.scale = p.scale;
    sp.out_bf16 = p.dtype == DSM_BF16;
    grid.x = static_cast<uint32_t>(rows < 512 ? rows : 512);
    return vec     ? launch_grid(k_orth_split<T, true, true>, grid, 256, 0, s, sp)
           : along ? launch_grid(k_orth_split<T, true, false>, grid, 256, 0, s, sp)
                   : launch_grid(k_orth_split<T, false, false>, grid, 256, 0, s, sp);
}

}  // namespace
}  // namespace ops
}  // namespace dsm

using namespace dsm;
using namespace dsm::ops;

extern "C" size_t dsm_orthogonalize_workspace(const dsm_orthogonalize_args* p) {
    if (check_args("dsm_orthogonalize_workspace", p) != DSM_OK) return 0;
    return make_plan(*p, nullptr).bytes;
}

extern "C" int dsm_orthogonalize(const dsm_orthogonalize_args* p, void* workspace, size_t workspace_bytes,
                                 dsm_stream_t stream) {
    if (int rc = check_args(kFunc, p); rc != DSM_OK) return rc;
    if (p->count == 0 || p->rows == 0 || p->cols == 0) return DSM_OK;
    if (!p->g || !p->out || !workspace) return fail(kFunc, DSM_EINVAL, "NULL argument");
    const uintptr_t esize = p->dtype == DSM_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(p->g) % esize || reinterpret_cast<uintptr_t>(p->out) % esize ||
        reinterpret_cast<uintptr_t>(p->momentum) % 4)
        return fail(kFunc, DSM_EALIGN, "g, out and momentum must be aligned to their elements");
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return fail(kFunc, DSM_EALIGN, "the workspace must be 256-byte aligned");
    Plan r = make_plan(*p, workspace);
    r.pairs = p->dtype == DSM_F32 ? p->steps : count_pairs(*p);
    if (workspace_bytes < r.bytes)
        return fail(kFunc, DSM_ENOMEM, "the workspace has %zu bytes, %llu are needed", workspace_bytes,
                    static_cast<unsigned long long>(r.bytes));
    int dev = 0, sms = 0;
    if (int rc = device_of_call(kFunc, &dev, &sms)) return rc;
    if (int rc = check_device(kFunc, p->g, "g", dev)) return rc;
    if (int rc = check_device(kFunc, p->out, "out", dev)) return rc;
    if (int rc = check_device(kFunc, workspace, "workspace", dev)) return rc;
    if (p->momentum)
        if (int rc = check_device(kFunc, p->momentum, "momentum", dev)) return rc;

    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint32_t* status = static_cast<uint32_t*>(workspace);
    const bool tall = r.rows > r.cols;
    if (const int cluster = p->dtype == DSM_BF16 ? small_cluster<__nv_bfloat16>(*p, r.m, tall ? r.rows : r.cols, dev, sms)
                                                 : small_cluster<float>(*p, r.m, tall ? r.rows : r.cols, dev, sms)) {
        auto turned = [&](const int64_t (&v)[3]) {
            const Strides o = r.oriented(v);
            return tall ? Strides{o.batch, o.col, o.row} : o;
        };
        SmallArgs a{};
        a.in.g = p->g;
        a.in.momentum = p->momentum;
        a.in.has_momentum = p->momentum != nullptr;
        a.in.status = status;
        a.in.gs = turned(p->g_stride);
        a.in.ms = turned(p->momentum_stride);
        a.in.rows = r.m;
        a.in.cols = tall ? r.rows : r.cols;
        a.in.mu = p->mu;
        a.in.nesterov = p->nesterov;
        a.out = p->out;
        a.os = turned(p->out_stride);
        const cudaError_t err = p->dtype == DSM_BF16 ? launch_small<__nv_bfloat16>(*p, a, cluster, s) : launch_small<float>(*p, a, cluster, s);
        return err == cudaSuccess ? DSM_OK : cuda_fail(kFunc, err, "launch the steps of small matrices");
    }
    const cudaError_t err = p->dtype == DSM_BF16 ? launch_start<__nv_bfloat16>(*p, r, status, s) : launch_start<float>(*p, r, status, s);
    if (err != cudaSuccess) return cuda_fail(kFunc, err, "launch the update");
    if (p->steps == 0) return DSM_OK;
    // Larger tiles read less, smaller ones keep more SMs at work.
    auto clocks = [&](uint32_t cg, uint32_t bn) { return step_clocks(r, p->count, sms, cg, bn, p->dtype == DSM_F32 ? 3 : 1); };
    const uint64_t c64 = clocks(1, 64), c128 = clocks(1, 128), p128 = clocks(2, 128);
    if (p->dtype == DSM_F32) {
        if (p128 <= c128 && p128 <= c64) return steps<2, 128, true>(*p, r, status, dev, s);
        return c128 <= c64 ? steps<1, 128, true>(*p, r, status, dev, s) : steps<1, 64, true>(*p, r, status, dev, s);
    }
    const uint64_t p256 = clocks(2, 256);
    if (p256 <= p128 && p256 <= c128 && p256 <= c64) return steps<2, 256, false>(*p, r, status, dev, s);
    if (p128 <= c128 && p128 <= c64) return steps<2, 128, false>(*p, r, status, dev, s);
    return c128 <= c64 ? steps<1, 128, false>(*p, r, status, dev, s) : steps<1, 64, false>(*p, r, status, dev, s);
}
