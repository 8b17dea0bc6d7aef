// dsm_orthogonalize for matrices with a side of at most 128: all of a call in one kernel, a cluster of CTAs to a matrix.
//
// A CTA keeps a slab of the columns of X (m x n, m <= 128) in shared memory, hi and lo.  Per step: its part of X X^T over
// the slab; the parts are added over the cluster through distributed shared memory, each CTA for its share of the rows,
// which it hands to all as A; then every CTA computes B = b A + c A A for itself and a X + B X for its slab.  The slab's
// layout (rows of 64 columns, 128-byte swizzle) is K-major to the first product and MN-major to the last, so X is never
// moved.  The steps touch no memory outside the SMs: two barriers of the cluster per step instead of three of the grid.
// Bound by the latency of that chain.
#pragma once

#include "orthogonalize.cuh"

namespace dsm {
namespace ops {
namespace {

struct SmallArgs {
    UpdateArgs in;               // rows = m <= cols
    void* out;
    Strides os;
    float eps, scale;
    uint32_t slab;               // columns of a CTA, a multiple of 64
    uint32_t steps;
    uint32_t gave_up;            // injected_timeout()
    float coefficients[3 * DSM_ORTHOGONALIZE_MAX_STEPS];
};

constexpr uint32_t kTile64 = 16384;      // 128 rows of 64 f16
template <typename T>
constexpr uint32_t small_tiles() {       // of a slab, at most: what fits next to A, B and the parts of A
    return sizeof(T) == 4 ? 3 : 4;
}
template <typename T>
__host__ __device__ constexpr uint32_t small_smem() {
    // X hi and lo; A (with 32-bit results hi and lo); the f32 part of A, whose place B takes after it
    return 2 * (sizeof(T) == 4 ? 3 : 4) * kTile64 + (sizeof(T) == 4 ? 4 : 2) * kTile64 + 4 * kTile64 + 1024;
}

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster2(uint32_t addr, uint2 v) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(addr), "r"(v.x), "r"(v.y) : "memory");
}
__device__ __forceinline__ uint16_t lds16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
    return v;
}

// Places in a matrix of 128 rows in tiles of 64 columns: of an element, and of the piece of 8 columns that holds column c.
__device__ __forceinline__ uint32_t small_piece(uint32_t r, uint32_t c) {
    return (c >> 6) * kTile64 + r * 128 + (((c >> 3 & 7) ^ (r & 7)) << 4);
}
__device__ __forceinline__ uint32_t small_place(uint32_t r, uint32_t c) { return small_piece(r, c) + (c & 7) * 2; }

template <typename T>
__global__ void __launch_bounds__(256, 1) k_orth_small(const __grid_constant__ SmallArgs p, uint32_t cluster) {
    constexpr bool kPair = sizeof(T) == 4;
    constexpr uint32_t kX = (kPair ? 3 : 4) * kTile64, kA = 2 * kTile64;
    extern __shared__ uint8_t raw[];
    __shared__ float2 sums[8], own_sum;
    __shared__ __align__(8) uint64_t done_bar;
    __shared__ uint32_t slot;
    const uint32_t x_hi = (smem_u32(raw) + 1023) & ~1023u, x_lo = x_hi + kX, a_hi = x_lo + kX, a_lo = a_hi + kA;
    const uint32_t part = a_hi + (kPair ? 2 : 1) * kA, b_hi = part, b_lo = part + kA;
    const uint32_t bar = smem_u32(&done_bar), tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const uint32_t rank = cluster > 1 ? cluster_rank() : 0;
    const UpdateArgs& in = p.in;
    const uint32_t m = in.rows, n = in.cols, c0 = rank * p.slab;
    const uint32_t mine = c0 >= n ? 0 : n - c0 < p.slab ? n - c0 : p.slab, tiles = p.slab / 64;
    const int64_t b = blockIdx.x / cluster;
    bool ok = !p.gave_up;        // of the warp

    if (tid == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc<1>(smem_u32(&slot), 512);
    for (uint32_t i = tid * 16; i < small_smem<T>() - 1024; i += 256 * 16) sts128(x_hi + i, uint4{});   // what lies beyond m and n
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = slot, d_gram = tmem, d_square = tmem + 128, d_apply = tmem + 256;
    wait_previous();
    if (blockIdx.x == 0 && tid == 0) *in.status = 0;

    // The slab's elements: a warp walks along rows or columns (`down`), whichever is closer together in memory, with every
    // 8th of the other; kBatch of a thread's elements at a time, all of whose loads are under way together (so none of
    // them may hang on a condition: beyond the end the last element is loaded again).
    constexpr int kBatch = 16;
    const T* g = static_cast<const T*>(in.g) + b * in.gs.batch + c0 * in.gs.col;
    float* mo = in.has_momentum ? in.momentum + b * in.ms.batch + c0 * in.ms.col : nullptr;
    auto walk = [&](bool down, auto&& batch) {
        const uint32_t fast = down ? m : mine, slow = down ? mine : m, along = (fast + 31) / 32;
        if (mine == 0) return;
        uint32_t i = warp, j = 0;
        while (i < slow) {
            uint32_t r[kBatch], c[kBatch];
            bool used[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const uint32_t f = j * 32 + lane;
                used[k] = i < slow && f < fast;
                const uint32_t sf = f < fast ? f : fast - 1, ss = i < slow ? i : slow - 1;
                r[k] = down ? sf : ss;
                c[k] = down ? ss : sf;
                if (++j == along) {
                    j = 0;
                    i += 8;
                }
            }
            batch(r, c, used);
        }
    };
    const bool down = mo ? llabs(in.ms.row) < llabs(in.ms.col) : llabs(in.gs.row) < llabs(in.gs.col);
    auto load = [&](const uint32_t (&r)[kBatch], const uint32_t (&c)[kBatch], float (&gv)[kBatch], float (&mv)[kBatch]) {
        T raw[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) raw[k] = g[r[k] * in.gs.row + c[k] * in.gs.col];
        if (mo) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) mv[k] = mo[r[k] * in.ms.row + c[k] * in.ms.col];
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) gv[k] = to_float(raw[k]);
    };
    float2 sum = make_float2(0.f, 0.f);
    walk(down, [&](const uint32_t (&r)[kBatch], const uint32_t (&c)[kBatch], const bool (&used)[kBatch]) {
        float gv[kBatch], mv[kBatch];
        load(r, c, gv, mv);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (!used[k]) continue;
            if (mo) {
                gv[k] = updated(in, gv[k], mv[k]);
                mo[r[k] * in.ms.row + c[k] * in.ms.col] = mv[k];
            }
            add_square(gv[k], sum);
        }
    });
    sum = cta_sum(sum, sums);
    if (cluster > 1) {
        if (tid == 0) own_sum = sum;
        cluster_sync();
        sum = make_float2(0.f, 0.f);
        for (uint32_t i = 0; i < cluster; ++i) {
            const uint32_t at = mapa(smem_u32(&own_sum), i);
            sum.x += ld_cluster(at);
            sum.y += ld_cluster(at + 4);
        }
    }
    const Unit unit = to_unit(sum, p.eps);
    // u again, from g and the new momentum (each thread its own)
    walk(down, [&](const uint32_t (&r)[kBatch], const uint32_t (&c)[kBatch], const bool (&used)[kBatch]) {
        float u[kBatch], mv[kBatch];
        load(r, c, u, mv);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (!used[k]) continue;
            if (mo) u[k] = in.nesterov ? fmaf(in.mu, mv[k], u[k]) : mv[k];
            __half hi, lo;
            split(unit(u[k]) * kScale, hi, lo);
            const uint32_t at = small_place(r[k], c[k]);
            sts16(x_hi + at, __half_as_ushort(hi));
            sts16(x_lo + at, __half_as_ushort(lo));
        }
    });

    // What all threads have written to shared memory is there for the matrix instructions, and what they have read of
    // tensor memory may be written.
    auto ready = [&](bool over_cluster) {
        if (over_cluster) asm volatile("fence.proxy.async;" ::: "memory");
        else fence_async_smem();
        tc_fence_before();
        if (over_cluster) {
            cluster_sync();
            asm volatile("fence.proxy.async;" ::: "memory");
        } else {
            __syncthreads();
        }
        tc_fence_after();
    };
    uint32_t phase = 0;
    // A product: D (128 x columns) over `blocks` of 16 k; the operands' places and steps per 16 k as functions.
    auto multiply = [&](uint32_t d, uint32_t idesc, uint32_t blocks, auto a_at, auto b_at, uint32_t a_plane, uint32_t b_plane, uint32_t lbo_b) {
        if (warp == 0 && ok) {   // (after a wait that ran out nothing more is multiplied)
            if (elect_one()) {
                constexpr int kTerms = kPair ? 3 : 1;
                for (uint32_t i = 0; i < blocks; ++i)
#pragma unroll
                    for (int term = 0; term < kTerms; ++term) {
                        const uint64_t da = smem_desc(a_at(i) + (kPair && term == 0 ? a_plane : 0), 16);
                        const uint64_t db = smem_desc(b_at(i) + (kPair && term == 1 ? b_plane : 0), lbo_b);
                        mma<1>(d, da, db, idesc, i > 0 || term > 0);
                    }
                mma_commit<1>(bar);
            }
            __syncwarp();
        }
        if (ok) ok = warp_wait(bar, phase);   // (who gave up goes on, so that the barriers meet, but waits no more)
        if (ok) phase ^= 1;
        __syncwarp();
        tc_fence_after();
    };
    const uint32_t row = warp % 4 * 32 + lane, half = warp / 4, lanes = (warp % 4 * 32) << 16;
    // What lies beyond m is zero, and stays so without being written (but for B in a cluster, whose place parts of A take).
    const bool beyond = warp % 4 * 32 >= m, idle = cluster == 1 && (beyond || half * 64 >= m);
    const uint32_t blocks_m = (m + 15) / 16;
    // 64 values of a thread's row of A or B, from column c, as hi and (32-bit results) lo
    auto store_row = [&](uint32_t hi, uint32_t lo, uint32_t c, const float (&v)[64]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint4 h = pack8<__half>(v + 8 * j);
            sts128(hi + small_piece(row, c + 8 * j), h);
            if constexpr (kPair) sts128(lo + small_piece(row, c + 8 * j), rest8<__half>(v + 8 * j, h));
        }
    };
    auto load_sums = [&](uint32_t d, uint32_t c, float (&v)[64]) {
        tmem_ld32(d + lanes + c, *reinterpret_cast<float(*)[32]>(v));
        tmem_ld32(d + lanes + c + 32, *reinterpret_cast<float(*)[32]>(v + 32));
        tmem_wait_ld();
    };
    ready(false);

    for (uint32_t k = 0; k < p.steps; ++k) {
        const float ca = p.coefficients[3 * k], cb = p.coefficients[3 * k + 1], cc = p.coefficients[3 * k + 2];
        __align__(16) float v[64];
        // A = X X^T
        auto x_k = [&](uint32_t i) { return x_hi + i / 4 * kTile64 + i % 4 * 32; };
        multiply(d_gram, instr_desc(false, false, false, 128, 128), tiles * 4, x_k, x_k, kX, kX, 16);
        if (!idle) load_sums(d_gram, half * 64, v);
        if (cluster == 1) {
            if (!idle) {
#pragma unroll
                for (int i = 0; i < 64; ++i) v[i] *= 1.f / kScale;
                store_row(a_hi, a_lo, half * 64, v);
            }
            ready(false);
        } else {
            // rows of 32 pieces of 16 bytes, the piece's place turned with the row
            auto piece = [&](uint32_t r, uint32_t j) { return part + r * 512 + ((j ^ (r & 7)) << 4); };
#pragma unroll
            for (int j = 0; j < 16; ++j) sts128(piece(row, half * 16 + j), *reinterpret_cast<uint4*>(v + 4 * j));
            cluster_sync();
            // The CTA's share of the rows: 16 pieces of all CTAs for every thread, loaded together; those of one place follow
            // each other.
            const uint32_t share = 128 / cluster, log2c = 31 - __clz(cluster);
            float4 x[16];
            auto at_r = [&](uint32_t i) { return rank * share + (tid + 256 * (i >> log2c)) / 32; };
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) {   // (what lies beyond m is zero and not asked for: 64 KB take 4000 clocks)
                x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (at_r(i) < m && 4 * lane < m) x[i] = ld_cluster4(mapa(piece(at_r(i), lane), i & (cluster - 1)));
            }
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) {
                s.x += x[i].x;
                s.y += x[i].y;
                s.z += x[i].z;
                s.w += x[i].w;
                if ((i + 1) & (cluster - 1)) continue;
                if (at_r(i) >= m || 4 * lane >= m) continue;
                const float e[4] = {s.x * (1.f / kScale), s.y * (1.f / kScale), s.z * (1.f / kScale), s.w * (1.f / kScale)};
                s = make_float4(0.f, 0.f, 0.f, 0.f);
                const uint2 hi = make_uint2(pack<__half>(e[0], e[1]), pack<__half>(e[2], e[3]));
                const float2 f0 = unpack<__half>(hi.x), f1 = unpack<__half>(hi.y);
                const uint2 lo = make_uint2(pack<__half>(e[0] - f0.x, e[1] - f0.y), pack<__half>(e[2] - f1.x, e[3] - f1.y));
                const uint32_t at = small_place(at_r(i), 4 * lane);
#pragma unroll 4
                for (uint32_t q = 0; q < cluster; ++q) {
                    st_cluster2(mapa(a_hi + at, q), hi);
                    if constexpr (kPair) st_cluster2(mapa(a_lo + at, q), lo);
                }
            }
            ready(true);
        }
        // B = b A + c A A
        auto a_k = [&](uint32_t i) { return a_hi + i / 4 * kTile64 + i % 4 * 32; };
        multiply(d_square, instr_desc(false, false, false, 128, 128), blocks_m, a_k, a_k, kA, kA, 16);
        if (!idle) load_sums(d_square, half * 64, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (idle) break;
            const uint4 h = lds128(a_hi + small_piece(row, half * 64 + 8 * j));
            const uint4 l = kPair ? lds128(a_lo + small_piece(row, half * 64 + 8 * j)) : uint4{};
            float a[8];
            unpack8<__half, kPair>(h, l, a);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[8 * j + q] = fmaf(cc * (1.f / kScale), v[8 * j + q], cb * a[q]);
        }
        if (!idle) store_row(b_hi, b_lo, half * 64, v);
        ready(false);
        // X <- a X + B X
        auto b_k = [&](uint32_t i) { return b_hi + i / 4 * kTile64 + i % 4 * 32; };
        auto x_mn = [&](uint32_t i) { return x_hi + i * 2048; };
        multiply(d_apply, instr_desc(false, false, true, 128, p.slab), blocks_m, b_k, x_mn, kA, kX, kTile64);
        const bool last = k + 1 == p.steps;
        for (uint32_t c = half * 64; c < p.slab && !beyond; c += 128) {
            load_sums(d_apply, c, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t at = small_piece(row, c + 8 * j);
                const uint4 h = lds128(x_hi + at), l = lds128(x_lo + at);
                float y[8];
                unpack8<__half, true>(h, l, y);
#pragma unroll
                for (int q = 0; q < 8; ++q) y[q] = fmaf(ca, y[q], v[8 * j + q] * (1.f / kScale));
                if (!last) {
                    const uint4 nh = pack8<__half>(y);
                    sts128(x_hi + at, nh);
                    sts128(x_lo + at, rest8<__half>(y, nh));
                    continue;
                }
                // the result: 16 bits in hi's place, 32 bits in both
#pragma unroll
                for (int q = 0; q < 8; ++q) y[q] *= p.scale / kScale;
                if constexpr (kPair) {
                    auto halves = [&](int q, bool upper) {
                        return __byte_perm(__float_as_uint(y[q]), __float_as_uint(y[q + 1]), upper ? 0x7632 : 0x5410);
                    };
                    sts128(x_hi + at, make_uint4(halves(0, true), halves(2, true), halves(4, true), halves(6, true)));
                    sts128(x_lo + at, make_uint4(halves(0, false), halves(2, false), halves(4, false), halves(6, false)));
                } else {
                    sts128(x_hi + at, pack8<__nv_bfloat16>(y));
                }
            }
        }
        ready(false);
    }

    T* out = static_cast<T*>(p.out) + b * p.os.batch;
    walk(llabs(p.os.row) < llabs(p.os.col), [&](const uint32_t (&r)[kBatch], const uint32_t (&c)[kBatch], const bool (&used)[kBatch]) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (!used[k]) continue;
            const uint32_t at = small_place(r[k], c[k]);
            const uint16_t hi = lds16(x_hi + at);
            T y;
            if constexpr (kPair) y = __uint_as_float(uint32_t(hi) << 16 | lds16(x_lo + at));
            else y = __ushort_as_bfloat16(hi);
            out[r[k] * p.os.row + (c0 + c[k]) * p.os.col] = y;
        }
    });
    if (!ok) {
        *in.status = 1;
        if (warp == 0) warp_wait(bar, phase);   // what it has issued may still be under way: shared and tensor memory are in use
    }
    tc_fence_before();
    const bool failed = __syncthreads_or(!ok);
    if (cluster > 1) cluster_sync();   // nobody reads this CTA's shared memory any more
    tc_fence_after();
    if (warp == 0) tmem_dealloc<1>(tmem, 512);
    // after all CTAs' results, which its own may have gone into
    if (failed) fill_nan(out, 1, m, n, 0, p.os.row, p.os.col, tid, 256);
}

// Whether a device takes clusters of 16 CTAs of the kernel.
template <typename T>
bool large_clusters(int dev) {
    static std::atomic<int> known[64];
    return most_clusters(k_orth_small<T>, 16, 256, small_smem<T>(), dev, known) > 0;
}

// The cluster's CTAs for matrices of m x n (m <= n), or 0 if they are not small: as many as share the columns in tiles of
// 64 while all matrices fit on the SMs at once, and at least as many as hold a matrix.  Large clusters that do not fit at
// once leave SMs idle, and the general way is faster.  This way and the general one, bf16 with momentum: 64 x 64 23 and 60 us,
// 200 of them 41 and 92, 2000 269 and 343; 128 x 1024 60 and 72, 24 of them 86 and 103; 10 of 95 x 3000 153 and 152; 24 of
// 128 x 4096 390 and 254.
template <typename T>
int small_cluster(const dsm_orthogonalize_args& p, uint32_t m, uint32_t n, int dev, int sms) {
    if (m > 128 || p.steps == 0) return 0;
    const uint32_t most = 64 * small_tiles<T>(), top = n > 8 * 64 && large_clusters<T>(dev) ? 16 : 8;
    uint32_t c = 1;
    while (c < top && c * most < n) c *= 2;
    if (c * most < n || (c >= 8 && uint64_t(c) * p.count > 2 * static_cast<uint64_t>(sms))) return 0;
    while (c < top && c * 64 < n && 2 * c * p.count <= static_cast<uint32_t>(sms)) c *= 2;
    return static_cast<int>(c);
}

template <typename T>
cudaError_t launch_small(const dsm_orthogonalize_args& p, SmallArgs& a, int cluster, cudaStream_t s) {
    auto kernel = k_orth_small<T>;
    a.eps = p.eps;
    a.scale = p.scale;
    a.slab = static_cast<uint32_t>(round_up(ceil_div(a.in.cols, cluster), 64));
    a.steps = p.steps;
    a.gave_up = injected_timeout();
    for (uint32_t i = 0; i < 3 * p.steps; ++i) a.coefficients[i] = p.coefficients[i];
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, small_smem<T>());
    if (err == cudaSuccess && cluster > 8) err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (err != cudaSuccess) return err;
    return launch_clusters(kernel, static_cast<int>(p.count) * cluster, cluster, 256, small_smem<T>(), s, true, a,
                           static_cast<uint32_t>(cluster));
}

}  // namespace
}  // namespace ops
}  // namespace dsm
