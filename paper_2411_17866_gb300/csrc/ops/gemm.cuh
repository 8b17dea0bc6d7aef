// The matrix product behind the operators: D = sum over terms of A B, f32 accumulators in tensor memory, an epilogue of
// the operator's own.  A is M x K and B is N x K; each lies K-major (k consecutive in memory) or MN-major.
//
// One persistent CTA per SM, or pairs of CTAs (CG = 2: one matrix instruction over both, 256 rows, each CTA with its half
// of the rows and loading its half of B).  Warps 0 and 2 load tiles of 64 k of A and B by TMA into a ring of stages, warp
// 1 issues the matrix instructions, the other warps read the finished accumulator and run the epilogue, while the other
// of the two accumulators is being filled.
//
// An epilogue warp has 32 rows and 64 or 128 columns of the tile.  In tensor memory a lane is a row, so a thread that
// wrote its row to global memory would touch 32 rows per instruction; what a warp reads and writes goes through a piece
// of shared memory of its own instead, 64 columns at a time, by TMA (Newton-Schulz on 24 x 1024 x 4096: a X + B X took
// 430 us with rows read and written by their threads).
//
// Three-term products (TERMS = 3): operands kept as pairs hi + lo of 16 bits multiply as lo B_hi + hi B_lo + hi B_hi, from
// one load of the four tiles.  What is left out (lo B_lo) is 2^-22 of the product in f16 and 2^-16 in bf16.  The tensor
// cores cut off what falls below the accumulator's last bit, which over a long K adds up to more than these products
// lose (f16 pairs, Newton-Schulz on 1024 x 4096: 3.6e-5 of the result after five steps).  With a CHUNK the accumulator
// is added to sums in registers after every CHUNK of k, rounded to nearest, and starts again from zero.
#pragma once

#include "dsm_device.cuh"
#include "tensor_core.cuh"

namespace dsm {
namespace ops {

constexpr int kBlockK = 64;      // k of one stage: one 128-byte swizzled row of 16-bit values
constexpr uint32_t kSmemMax = 227 * 1024;

// Work of one launch, in tiles of BM x BN.
struct Schedule {
    uint32_t tiles_m, tiles_n, batches;
    uint32_t splits;             // parts of K, each a tile of its own
    uint32_t k;                  // in all
    uint32_t symmetric;          // only tiles on or above the diagonal (in squares of max(BM, BN)); tiles_m, tiles_n count those
    uint32_t n_fast;             // neighbouring tiles differ in n (else in m)
    const uint32_t* m_count;     // device memory: rows of M in use (or null)
    const uint32_t* k_count;     // device memory: k in use (or null)
    const uint32_t* split_count; // device memory: in place of `splits` (or null)
    uint32_t* status;            // set to 1 if a wait ran out
};

struct Maps {
    CUtensorMap a[2], b[2];      // hi, lo
};

struct Tile {
    uint32_t m0, n0, batch, split;
    uint32_t k0, k1;             // blocks of k, a stage each: none if k0 = k1 (the accumulator is then zero)
};

// CHUNK: k between two additions to sums in registers; 0: none.
template <int CG_, int BN_, int TERMS_, uint32_t CHUNK, bool BF16_, uint32_t BUFFER>
struct Shape {
    static constexpr int CG = CG_, BN = BN_, TERMS = TERMS_;
    static constexpr bool CHUNKED = CHUNK > 0, BF16 = BF16_;
    static constexpr int kPair = TERMS == 3 ? 2 : 1;
    // Blocks of 64 k per stage: two where issuing takes longer than multiplying (waits are per stage).
    static constexpr uint32_t kSub = CG == 1 && TERMS == 1 && BN <= 128 ? 2 : 1;
    static constexpr uint32_t kChunk = CHUNK / (kBlockK * kSub);   // stages between two additions to the register sums
    static_assert(kChunk * kBlockK * kSub == CHUNK, "whole stages");
    static constexpr int kEpiWarps = BN == 64 ? 4 : 8;
    static constexpr int kFirstEpi = 3;                                             // warps before the epilogue's
    static constexpr int kThreads = 32 * (kFirstEpi + kEpiWarps);
    static constexpr int kWarpColumns = BN * 4 / kEpiWarps;
    static constexpr uint32_t kA = 128 * kBlockK * 2, kB = BN / CG * kBlockK * 2;   // bytes of one operand's tile
    static constexpr uint32_t kStage = kSub * kPair * (kA + kB);                    // A's tiles, then B's
    static constexpr uint32_t kBuffer = BUFFER, kBuffers = kEpiWarps * BUFFER;                 // the epilogue's shared memory
    static constexpr uint32_t kFit = (kSmemMax - 2048 - kBuffers) / kStage;
    static constexpr uint32_t kStages = kFit < 12 ? kFit : 12;
    static constexpr uint32_t kSmem = kStages * kStage + kBuffers + 2048;           // 1024 for alignment, 1024 for barriers
    // Accumulators: with sums in registers as many as tensor memory holds (they are small turns: while a tile is stored the
    // next one's first ones are multiplied; 1024 tokens on 50257 x 768 f32: loss 218 us with two, 204 with four).
    static constexpr uint32_t kAcc = CHUNKED && BN == 128 ? 4 : 2;
    static constexpr uint32_t kColumns = kAcc * BN;                                 // of tensor memory
    static_assert(BN == 64 || BN == 128 || BN == 256, "tile shape");
    static_assert(kStages >= 2 && BUFFER % 1024 == 0 && (2 * kStages + 2 * kAcc + kEpiWarps + 8) * 8 <= 1024, "shared memory");
};

template <class S>
struct Scheduler {
    uint32_t tiles, tiles_m, tiles_n, per, kblocks, splits, symmetric, n_fast;
    static constexpr uint32_t BM = 128 * S::CG, BN = S::BN, kBlock = kBlockK * S::kSub;
    static constexpr uint32_t kG = BM > BN ? BM : BN;
    static constexpr uint32_t kSub = (kG / BM) * (kG / BN);

    __device__ explicit Scheduler(const Schedule& s)
        : tiles_m(s.tiles_m), tiles_n(s.tiles_n), splits(s.splits), symmetric(s.symmetric), n_fast(s.n_fast) {
        uint32_t k = s.k;
        if (s.m_count) {
            const uint32_t used = (*s.m_count + BM - 1) / BM;
            tiles_m = used < tiles_m ? used : tiles_m;
        }
        if (s.k_count) k = *s.k_count < k ? *s.k_count : k;
        if (s.split_count) splits = *s.split_count;
        kblocks = (k + kBlock - 1) / kBlock;
        per = symmetric ? tiles_m * (tiles_m + 1) / 2 * kSub : tiles_m * tiles_n * splits;
        tiles = per * s.batches;
    }

    __device__ Tile at(uint32_t t) const {
        Tile r;
        r.batch = t / per;
        t -= r.batch * per;
        if (symmetric) {  // rows of squares: square (i, j), j >= i
            const uint32_t sub = t % kSub;
            t /= kSub;
            uint32_t i = 0, left = tiles_m;
            while (t >= left) {
                t -= left;
                ++i;
                --left;
            }
            r.m0 = i * kG + sub / (kG / BN) * BM;
            r.n0 = (i + t) * kG + sub % (kG / BN) * BN;
            r.split = 0;
            r.k0 = 0;
            r.k1 = kblocks;
            return r;
        }
        r.split = t % splits;
        t /= splits;
        const uint32_t m = n_fast ? t / tiles_n : t % tiles_m, n = n_fast ? t % tiles_n : t / tiles_m;
        r.m0 = m * BM;
        r.n0 = n * BN;
        r.k0 = static_cast<uint32_t>(uint64_t(kblocks) * r.split / splits);
        r.k1 = static_cast<uint32_t>(uint64_t(kblocks) * (r.split + 1) / splits);
        return r;
    }
};


// An epilogue warp's shared memory and the barrier of its loads.
struct WarpBuffer {
    uint32_t addr, bar, loads;
    uint32_t lane, columns;   // columns: of the warp in a tile
    __device__ __forceinline__ bool wait_load() {
        const bool done = warp_wait(bar, loads & 1);
        ++loads;
        return done;
    }
    // The buffer as 32 rows of 128 bytes in TMA's 128-byte swizzle, a thread to a row; piece j of 16 bytes.
    __device__ __forceinline__ uint32_t at(int j) const { return addr + lane * 128 + ((j ^ (lane & 7)) << 4); }
    // Stores that have been started no longer read the buffer.
    __device__ __forceinline__ void reuse() const {
        if (lane == 0) tma_store_wait_read();
        __syncwarp();
    }
    // What the warp has written to the buffer can be stored; true in the thread that does it.
    __device__ __forceinline__ bool written() const {
        fence_async_smem();
        __syncwarp();
        return lane == 0;
    }
};

// Whether TMA may store a box that ends at column `end` of rows of `cols` columns of the caller's: it writes whole pieces of 16
// bytes, the one with a row's last column too, and what lies behind that is not the operator's.
template <typename T>
__device__ __forceinline__ bool ends_whole(uint32_t end, uint32_t cols) {
    return end <= cols || cols % (16 / sizeof(T)) == 0;
}

// Stores every STEP'th of a buffer's 32 rows of 64 16-bit values, from row `first` on, two values at a time.  ODD: rows that
// start in the middle of a word; the first and the last value are then stored alone.
template <bool ODD, int STEP>
__device__ __forceinline__ void store_words(uint32_t addr, uint32_t lane, uint16_t* to, int64_t rs, uint32_t first) {
    constexpr int kBatch = 8;
    to += first * rs + 2 * lane + ODD;
    const uint32_t place = lane * 4;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += kBatch * STEP) {
        uint32_t own[kBatch], next[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t r = first + r0 + i * STEP;
            own[i] = lds<uint32_t>(addr + r * 128 + (place ^ (r & 7) << 4));
        }
        if constexpr (ODD)
#pragma unroll
            for (int i = 0; i < kBatch; ++i) next[i] = __shfl_down_sync(0xffffffffu, own[i], 1);
#pragma unroll
        for (int i = 0; i < kBatch; ++i, to += STEP * rs) {
            if constexpr (!ODD) {
                *reinterpret_cast<uint32_t*>(to) = own[i];
            } else {
                const uint32_t two = __funnelshift_r(own[i], next[i], 16);
                if (lane < 31) *reinterpret_cast<uint32_t*>(to) = two;
                if (lane == 31) *to = static_cast<uint16_t>(two);
                if (lane == 0) to[-1] = static_cast<uint16_t>(own[i]);
            }
        }
    }
}

// Plain stores of a buffer's 32 rows of 128 bytes (at `addr`), neighbouring threads on neighbouring columns: `rows` x `cols`
// of it, to rows and columns rs and cs elements apart.  Bound by its instructions (dW of 25 tokens on 50257 x 1102: 47 us
// with one 16-bit value at a time, 34 with two; by TMA, where rows start on 16-byte boundaries, 25).
template <typename T>
__device__ __forceinline__ void store_box(uint32_t addr, uint32_t lane, T* to, int64_t rs, int64_t cs, uint32_t rows, uint32_t cols) {
    constexpr uint32_t kCols = 128 / sizeof(T);
    if constexpr (sizeof(T) == 2) {
        if (cs == 1 && rows >= 32 && cols >= kCols) {
            uint16_t* row = reinterpret_cast<uint16_t*>(to);
            const uint32_t odd = reinterpret_cast<uintptr_t>(row) / 2 & 1;
            if (rs & 1) {
                store_words<false, 2>(addr, lane, row, rs, odd);
                store_words<true, 2>(addr, lane, row, rs, odd ^ 1);
            } else if (odd) {
                store_words<true, 1>(addr, lane, row, rs, 0);
            } else {
                store_words<false, 1>(addr, lane, row, rs, 0);
            }
            return;
        }
    }
    const uint32_t last = rows < 32 ? rows : 32;
#pragma unroll 4
    for (uint32_t r = 0; r < last; ++r)
#pragma unroll
        for (uint32_t c = lane; c < kCols; c += 32) {
            const uint32_t byte = c * sizeof(T);
            if (c < cols) to[r * rs + c * cs] = lds<T>(addr + r * 128 + ((byte / 16 ^ (r & 7)) << 4) + byte % 16);
        }
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T round_to(float v);
template <>
__device__ __forceinline__ float round_to<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half round_to<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 round_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <typename T>
__device__ __forceinline__ void split(float v, T& hi, T& lo) {
    hi = round_to<T>(v);
    lo = round_to<T>(v - to_float(hi));
}

// Two values as one word, the first in its lower half, and back: one instruction each way (arrays of 16-bit values cost
// several for every value).
template <typename T>
__device__ __forceinline__ uint32_t pack(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack<__half>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ float2 unpack(uint32_t v);
template <>
__device__ __forceinline__ float2 unpack<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
template <>
__device__ __forceinline__ float2 unpack<__nv_bfloat16>(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
// 8 values rounded, and what rounding leaves of them.
template <typename T>
__device__ __forceinline__ uint4 pack8(const float* v) {
    return make_uint4(pack<T>(v[0], v[1]), pack<T>(v[2], v[3]), pack<T>(v[4], v[5]), pack<T>(v[6], v[7]));
}
template <typename T>
__device__ __forceinline__ uint4 rest8(const float* v, const uint4& hi) {
    auto rest = [&](int i, uint32_t h) {
        const float2 f = unpack<T>(h);
        return pack<T>(v[i] - f.x, v[i + 1] - f.y);
    };
    return make_uint4(rest(0, hi.x), rest(2, hi.y), rest(4, hi.z), rest(6, hi.w));
}
// 8 values from hi and (with PAIR) lo.
template <typename T, bool PAIR>
__device__ __forceinline__ void unpack8(const uint4& hi, const uint4& lo, float (&v)[8]) {
    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 f = unpack<T>(h[i]);
        if constexpr (PAIR) {
            const float2 r = unpack<T>(l[i]);
            f.x += r.x;
            f.y += r.y;
        }
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// What an epilogue reads its 32 columns from, c = 0, 32, ...: tensor memory, or the sums in registers (whose loop over c
// has to be unrolled).
template <class Release>
struct TmemColumns {
    static constexpr int kUnroll = 1;
    uint32_t addr;
    Release& release;
    __device__ __forceinline__ void load(int c, float (&v)[32]) const {
        tmem_ld32(addr + c, v);
        tmem_wait_ld();
    }
    __device__ __forceinline__ void done() const { release(); }
};
template <int BN>
struct RegisterColumns {
    static constexpr int kUnroll = BN / 32;
    const float (&sum)[BN];
    __device__ __forceinline__ void done() const {}
    __device__ __forceinline__ void load(int c, float (&v)[32]) const {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = sum[c + k];
    }
};

// A CTA's pipeline: its shared memory, its barriers, and how far each of its roles has come.
template <class S>
struct Pipe {
    uint32_t base, buffers, bars, tmem;
    uint32_t warp, lane, rank, unit, units;
    uint32_t it = 0, turn = 0;   // stages and accumulators, as counted by the role that this thread has
    WarpBuffer buf;
    bool ok = true;

    __device__ __forceinline__ uint32_t full(uint32_t s) const { return bars + 8 * s; }
    __device__ __forceinline__ uint32_t empty(uint32_t s) const { return bars + 8 * (S::kStages + s); }
    __device__ __forceinline__ uint32_t acc_full(uint32_t s) const { return bars + 8 * (2 * S::kStages + s); }
    __device__ __forceinline__ uint32_t acc_empty(uint32_t s) const { return acc_full(S::kAcc + s); }
    __device__ __forceinline__ uint32_t drain() const { return acc_full(2 * S::kAcc); }
    __device__ __forceinline__ uint32_t slot() const { return acc_full(2 * S::kAcc + 1); }
    __device__ __forceinline__ uint32_t go() const { return acc_full(2 * S::kAcc + 2); }
    __device__ __forceinline__ uint32_t done_warps() const { return acc_full(2 * S::kAcc + 3); }
    __device__ __forceinline__ uint32_t load_bar(uint32_t w) const { return acc_full(2 * S::kAcc + 4 + w); }
    // The accumulator of the current turn, and its turn's parity.
    __device__ __forceinline__ uint32_t acc() const { return turn % S::kAcc; }
    __device__ __forceinline__ uint32_t acc_parity() const { return turn / S::kAcc & 1; }

    // The producers and the multiplier are one thread each, elected by its warp with elect.sync: the compiler then keeps
    // descriptors in the uniform registers that the instructions take.  (A thread picked by its index took 590 clocks to
    // issue a block of 64 k, a whole warp in step that elects a thread per block 320; 128 x 64 x 64 multiplies in 128.)
    __device__ __forceinline__ bool producer_a() const { return warp == 0; }
    __device__ __forceinline__ bool producer_b() const { return warp == 2; }
    __device__ __forceinline__ bool multiplier() const { return warp == 1 && rank == 0; }
    __device__ __forceinline__ bool finisher() const { return warp >= S::kFirstEpi; }

    __device__ __forceinline__ void open(uint8_t* raw) {
        base = (smem_u32(raw) + 1023) & ~1023u;
        buffers = base + S::kStages * S::kStage;
        bars = buffers + S::kBuffers;
        warp = threadIdx.x / 32;
        lane = threadIdx.x % 32;
        rank = S::CG == 2 ? cluster_rank() : 0;
        unit = blockIdx.x / S::CG;
        units = gridDim.x / S::CG;
        const uint32_t epi = warp - S::kFirstEpi;
        if (finisher()) buf = WarpBuffer{buffers + epi * S::kBuffer, load_bar(epi), 0, lane, S::kWarpColumns};
        if (threadIdx.x == 0) {
            for (uint32_t s = 0; s < S::kStages; ++s) {
                mbar_init(full(s), 2);   // A and B
                mbar_init(empty(s), 1);
            }
            for (uint32_t s = 0; s < S::kAcc; ++s) {
                mbar_init(acc_full(s), 1);
                mbar_init(acc_empty(s), S::kEpiWarps * S::CG);
            }
            mbar_init(drain(), 1);
            mbar_init(go(), 1);
            for (uint32_t w = 0; w < S::kEpiWarps; ++w) mbar_init(load_bar(w), 1);
            asm volatile("st.shared.u32 [%0], 0;" ::"r"(done_warps()) : "memory");
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        if (warp == 1) tmem_alloc<S::CG>(slot(), S::kColumns);
        tc_fence_before();
        sync();
        tc_fence_after();
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot()));
    }
    __device__ __forceinline__ void sync() const {
        if constexpr (S::CG == 2) cluster_sync();
        else __syncthreads();
    }
    // After the elected thread's part of a product: its state, in all threads of the warp.
    __device__ __forceinline__ void meet() {
        __syncwarp();
        ok = __all_sync(0xffffffffu, ok);
        it = __reduce_max_sync(0xffffffffu, it);
        turn = __reduce_max_sync(0xffffffffu, turn);
    }
    // Ends the CTA's (or pair's) work.  In a run that gave up nothing may be under way: neither copies nor instructions.
    __device__ __forceinline__ void close(uint32_t* status) {
        if (!ok) {
            *status = 1;
            if ((producer_a() || producer_b()) && rank == 0)
                for (uint32_t i = it > S::kStages ? it - S::kStages : 0; i < it; ++i)
                    mbar_wait(full(i % S::kStages), i / S::kStages & 1);
            if (multiplier()) {
                if (elect_one()) mma_commit<S::CG>(drain());
                __syncwarp();
                mbar_wait(drain(), 0);
            }
            if (finisher()) mbar_wait(buf.bar, buf.loads & 1);
        }
        if (finisher()) tma_store_wait();
        __syncwarp();
        tc_fence_before();
        sync();
        tc_fence_after();
        if (warp == 1) tmem_dealloc<S::CG>(tmem, S::kColumns);
    }
};

// Accumulators are handed over in turns: one turn is a tile, or with a CHUNK that part of its k (one turn at least).
template <class S>
__device__ __forceinline__ uint32_t turn_end(const Tile& w, uint32_t k) {
    return !S::CHUNKED || w.k1 - k <= S::kChunk ? w.k1 : k + S::kChunk;
}

// A producer's part of a product: its operand in every stage of every tile.  One thread.
template <bool IS_B, bool MN, class S, class Sched>
__device__ __forceinline__ void produce(Pipe<S>& p, const CUtensorMap (&maps)[2], const Sched& sched) {
    constexpr int kRows = IS_B ? S::BN / S::CG : 128;
    constexpr uint32_t kBytes = IS_B ? S::kB : S::kA;
    const uint32_t first = p.base + (IS_B ? S::kSub * S::kPair * S::kA : 0);
    const uint32_t bars = S::CG == 2 ? mapa(p.full(0), 0) : p.full(0);   // of the pair's first CTA
    uint32_t s = p.it % S::kStages, ph = p.it / S::kStages & 1;
    for (uint32_t t = p.unit; t < sched.tiles; t += p.units) {
        const Tile w = sched.at(t);
        const int x = static_cast<int>((IS_B ? w.n0 : w.m0) + p.rank * kRows), z = static_cast<int>(w.batch);
        for (uint32_t k = w.k0; k < w.k1; ++k) {
            if (!(p.ok = mbar_wait(p.empty(s), ph ^ 1))) return;
            if (p.rank == 0) mbar_expect(p.full(s), S::CG * S::kSub * S::kPair * kBytes);
            const uint32_t to = first + s * S::kStage, bar = bars + 8 * s;
#pragma unroll
            for (uint32_t i = 0; i < S::kSub * S::kPair; ++i) {   // (what lies beyond the last k reads as zero)
                const int kx = static_cast<int>((k * S::kSub + i / S::kPair) * kBlockK);
                const CUtensorMap* map = &maps[i % S::kPair];
                if constexpr (MN) {
#pragma unroll
                    for (int j = 0; j < kRows / 64; ++j)
                        tma_load<S::CG>(to + i * kBytes + j * 8192, map, bar, x + 64 * j, kx, z);
                } else {
                    tma_load<S::CG>(to + i * kBytes, map, bar, kx, x, z);
                }
            }
            ++p.it;
            if (++s == S::kStages) {
                s = 0;
                ph ^= 1;
            }
        }
    }
}

// The matrix instructions of a product.  One thread.
template <bool A_MN, bool B_MN, class S, class Sched>
__device__ __forceinline__ void multiply(Pipe<S>& p, const Sched& sched) {
    constexpr uint32_t kIdesc = instr_desc(S::BF16, A_MN, B_MN, 128 * S::CG, S::BN);
    static_assert(!B_MN || S::BN / S::CG % 64 == 0, "tile shape");
    // of the first stage; further ones and further k are added to its address field
    const uint64_t a0 = smem_desc(p.base, A_MN ? 8192 : 16), 
                   b0 = smem_desc(p.base + S::kSub * S::kPair * S::kA, B_MN ? 8192 : 16);
    uint32_t s = p.it % S::kStages, ph = p.it / S::kStages & 1;
    for (uint32_t t = p.unit; t < sched.tiles; t += p.units) {
        const Tile w = sched.at(t);
        uint32_t k = w.k0;
        do {
            const uint32_t d = p.acc(), end = turn_end<S>(w, k);
            if (!(p.ok = mbar_wait(p.acc_empty(d), p.acc_parity() ^ 1))) return;
            tc_fence_after();
            const uint32_t acc = p.tmem + d * S::BN;
            for (uint32_t first = k; k < end; ++k, ++p.it) {
                if (!(p.ok = mbar_wait(p.full(s), ph))) return;
                tc_fence_after();
                const uint64_t a = a0 + s * (S::kStage >> 4), b = b0 + s * (S::kStage >> 4);
#pragma unroll
                for (uint32_t part = 0; part < S::kSub * S::TERMS; ++part) {
                    const uint32_t term = part % S::TERMS, sub = part / S::TERMS * S::kPair;
                    // three terms: (lo, hi), (hi, lo), (hi, hi); one term: (hi, hi)
                    const uint64_t at = a + ((sub + (S::TERMS == 3 && term == 0)) * S::kA >> 4);
                    const uint64_t bt = b + ((sub + (S::TERMS == 3 && term == 1)) * S::kB >> 4);
#pragma unroll
                    for (int i = 0; i < kBlockK / 16; ++i)
                        // the next 16 k: 32 bytes along a K-major row, 16 rows of 128 bytes down an MN-major tile
                        mma<S::CG>(acc, at + (A_MN ? i * 128 : i * 2), bt + (B_MN ? i * 128 : i * 2), kIdesc,
                                   k > first || part > 0 || i > 0);
                }
                mma_commit<S::CG>(p.empty(s));
                if (++s == S::kStages) {
                    s = 0;
                    ph ^= 1;
                }
            }
            mma_commit<S::CG>(p.acc_full(d));
            ++p.turn;
        } while (k < w.k1);
    }
}

// The epilogue of a product.  Epi: struct with
//   static constexpr uint32_t kBuffer               bytes of shared memory per epilogue warp, a multiple of 1024
//   before(t, row, col, buf)                        ahead of the wait for the accumulator: starts loads
//   bool tile<COLUMNS>(t, row, col, acc, empty, buf)
// called by every thread of the epilogue warps.  (row, col): the warp's first row of M and column of N.  `empty`: K is
// empty, what acc gives has no meaning (the product is zero).  tile() calls acc.done() after its last load, if there is one
// (the accumulator is then free for the next product), and returns false if a wait ran out.
template <class S, class Sched, class Epi>
__device__ __forceinline__ void finish(Pipe<S>& p, const Sched& sched, const Epi& epi) {
    constexpr int kCols = S::kWarpColumns;
    const uint32_t quarter = p.warp % 4, part = (p.warp - S::kFirstEpi) / 4;   // the warp's lanes and columns
    auto acquire = [&] {
        p.ok = warp_wait(p.acc_full(p.acc()), p.acc_parity());
        tc_fence_after();
        return p.ok;
    };
    uint32_t released = 0;
    auto release = [&] {
        if (released == p.turn + 1) return;
        released = p.turn + 1;
        tc_fence_before();
        __syncwarp();
        if (p.lane == 0) {
            if constexpr (S::CG == 2) mbar_arrive_cluster(mapa(p.acc_empty(p.acc()), 0));
            else mbar_arrive(p.acc_empty(p.acc()));
        }
    };
    for (uint32_t t = p.unit; t < sched.tiles; t += p.units) {
        const Tile w = sched.at(t);
        const uint32_t row = w.m0 + p.rank * 128 + quarter * 32, col = w.n0 + part * kCols;
        const uint32_t lanes = p.tmem + (quarter * 32 << 16) + part * kCols;
        epi.before(w, row, col, p.buf);
        if constexpr (!S::CHUNKED) {
            if (!acquire()) return;
            p.ok = epi.template tile<kCols>(w, row, col, TmemColumns<decltype(release)>{lanes + p.acc() * S::BN, release},
                                             w.k0 == w.k1, p.buf);
            release();
            ++p.turn;
        } else {
            float sum[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) sum[c] = 0.f;
            uint32_t k = w.k0;
            do {
                if (!acquire()) return;
                const TmemColumns<decltype(release)> acc{lanes + p.acc() * S::BN, release};
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                    float v[32];
                    acc.load(c, v);
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum[c + i] += v[i];
                }
                release();
                ++p.turn;
                k = turn_end<S>(w, k);
            } while (k < w.k1);
            p.ok = epi.template tile<kCols>(w, row, col, RegisterColumns<kCols>{sum}, w.k0 == w.k1, p.buf);
        }
        if (!p.ok) return;
    }
}

// One product as a kernel.
template <class S, bool A_MN, bool B_MN, class Epi>
__global__ void __launch_bounds__(S::kThreads, 1)
k_gemm(const __grid_constant__ Maps maps, const __grid_constant__ Schedule work, const __grid_constant__ Epi epi) {
    extern __shared__ uint8_t raw[];
    if (threadIdx.x == 0) {
        prefetch_map(&maps.a[0]);
        prefetch_map(&maps.b[0]);
    }
    Pipe<S> p;
    p.open(raw);
    wait_previous();
    const Scheduler<S> sched(work);
    if (p.producer_a()) {
        if (elect_one()) produce<false, A_MN>(p, maps.a, sched);
        p.meet();
    } else if (p.producer_b()) {
        if (elect_one()) produce<true, B_MN>(p, maps.b, sched);
        p.meet();
    } else if (p.multiplier()) {
        if (elect_one()) multiply<A_MN, B_MN>(p, sched);
        p.meet();
    } else if (p.finisher()) {
        finish(p, sched, epi);
    }
    p.close(work.status);
}

// All CTAs of a cooperative launch, between two of its products.  What the epilogue warps have stored by TMA is arrived
// with (plain stores would need a fence to come before the TMA loads of other CTAs: 1 us); threads that go on to read it
// wait.
struct GridBarrier {
    uint32_t* count;             // zero at the launch: CTAs that are done with a product, of all products
    uint32_t phase = 0;
    // By the epilogue warps, each as it gets done: the last of a CTA's `warps` arrives.  Nothing waits here, so that a warp
    // that gave up holds up nobody.
    __device__ __forceinline__ void arrive(uint32_t done_warps, uint32_t warps) const {
        __syncwarp();
        if (threadIdx.x % 32 == 0) {  // the thread that stores
            tma_store_wait();
            uint32_t before;
            asm volatile("atom.acq_rel.cta.shared::cta.add.u32 %0, [%1], 1;" : "=r"(before) : "r"(done_warps) : "memory");
            if (before % warps == warps - 1) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(count) : "memory");
        }
        __syncwarp();
    }
    // Until `ctas` CTAs are done with all products so far; false if that takes longer than kWaitClocks.
    __device__ __forceinline__ bool wait(uint32_t ctas) const {
        const uint32_t want = ctas * phase;
        uint32_t seen = 0;
        const long long began = clock64();
        do {
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(count) : "memory");
            if (seen >= want) {
                asm volatile("fence.proxy.async;" ::: "memory");
                return true;
            }
        } while (clock64() - began < kWaitClocks);
        return false;
    }
};

}  // namespace ops
}  // namespace dsm
