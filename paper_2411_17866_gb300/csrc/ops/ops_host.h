// Host side shared by the operators: errors, device checks, tensor maps, launches of the matrix product.
#pragma once

#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include <cuda.h>
#include <cuda_runtime.h>

#include "dsm.h"
#include "dsm_internal.h"
#include "gemm.cuh"

namespace dsm {
namespace ops {

// Every workspace starts with its status word (0, or 1 after a wait that ran out).
constexpr uint64_t kHeaderBytes = 256;

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
inline uint32_t ceil_div(uint64_t v, uint64_t by) { return static_cast<uint32_t>((v + by - 1) / by); }

inline int fail(const char* func, int code, const char* fmt, ...) {
    char msg[400], buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    snprintf(buf, sizeof buf, "%s: %s", func, msg);
    set_last_error_message(buf);
    return code;
}

inline int cuda_fail(const char* func, cudaError_t e, const char* what) {
    cudaGetLastError();  // reported here: it must not be found again by a later call's check
    return fail(func, DSM_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

// DSM_INJECT_OPERATOR_TIMEOUT=1: kernels that wait act as if a wait of theirs had run out (fault injection for tests).
inline bool injected_timeout() {
    const char* inject = std::getenv("DSM_INJECT_OPERATOR_TIMEOUT");
    return inject && inject[0] == '1';
}

// Hands out consecutive 256-byte aligned pieces; with a null base it only adds up the size.
struct Carver {
    uint8_t* base;
    uint64_t used;
    explicit Carver(void* p) : base(static_cast<uint8_t*>(p)), used(kHeaderBytes) {}
    template <typename T>
    T* take(uint64_t count) {
        const uint64_t at = used;
        used += round_up(count * sizeof(T), 256);
        return base ? reinterpret_cast<T*>(base + at) : nullptr;
    }
};

// NaN in all places of `count` matrices of rows x cols, by the threads `first`, first + step, ...: what becomes of results after
// a wait that ran out.
template <typename T>
__device__ inline void fill_nan(T* to, uint64_t count, uint64_t rows, uint64_t cols, int64_t matrix, int64_t row, int64_t col,
                                uint64_t first, uint64_t step) {
    for (uint64_t i = first; i < count * rows * cols; i += step) {
        const uint64_t r = i / cols;
        to[int64_t(r / rows) * matrix + int64_t(r % rows) * row + int64_t(i % cols) * col] = round_to<T>(NAN);
    }
}

int check_device(const char* func, const void* p, const char* name, int dev);
int device_of_call(const char* func, int* dev, int* sms);

enum class Elem { f16, bf16, f32 };

// A 3-D tensor map with the 128-byte swizzle: (x, y, z) of the sizes nx, ny, nz; rows of `ld` elements, planes of
// `plane` elements; a box of 128 bytes x rows x 1.  What lies outside reads as zero and is not written (but in pieces of
// 16 bytes: see tma_store).
int make_map(const char* func, CUtensorMap* map, const void* base, uint64_t nx, uint64_t ny, uint64_t nz, uint64_t ld,
             uint64_t plane, uint32_t rows, Elem type);
// The same without a swizzle and with boxes of 64 bytes x rows x 1.
int make_plain_map(const char* func, CUtensorMap* map, const void* base, uint64_t nx, uint64_t ny, uint64_t nz, uint64_t ld,
                   uint64_t plane, uint32_t rows, Elem type);

// Whether make_map() takes a buffer of the caller's: addresses, rows and planes (of more than one) on 16 bytes.
inline bool mappable(const void* base, int64_t ld, int64_t plane, uint64_t ny, uint64_t nz, int esize) {
    auto fits = [&](int64_t stride) { return stride > 0 && stride * esize % 16 == 0 && stride * esize < (int64_t(1) << 40); };
    return reinterpret_cast<uintptr_t>(base) % 16 == 0 && (ny <= 1 || fits(ld)) && (nz <= 1 || fits(plane));
}

// A dependent launch (wait_previous()) on a grid of up to three dimensions.
template <typename... Params, typename... Args>
cudaError_t launch_grid(void (*kernel)(Params...), dim3 grid, uint32_t threads, size_t smem, cudaStream_t s,
                        const Args&... args) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

// The most clusters of CTAs of a kernel that a device runs at the same time; 0 if it takes none.  A property of the kernel
// and the device, asked for once: `known` holds the answer + 1 by device.
template <typename Kernel>
int most_clusters(Kernel kernel, int cluster, uint32_t threads, size_t smem, int dev, std::atomic<int> (&known)[64]) {
    if (dev >= 0 && dev < 64)
        if (const int k = known[dev].load()) return k - 1;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = static_cast<unsigned>(cluster);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(cluster));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int count = 0;
    const bool fits = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) == cudaSuccess &&
                      (cluster <= 8 || cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) &&
                      cudaOccupancyMaxActiveClusters(&count, kernel, &cfg) == cudaSuccess;
    cudaGetLastError();  // an answer of none is no error to be found by a later call
    if (!fits) count = 0;
    if (dev >= 0 && dev < 64) known[dev].store(count + 1);
    return count;
}

// A cooperative launch of up to `clusters` clusters, but no more than run at the same time.
template <typename... Params, typename... Args>
cudaError_t launch_together(void (*kernel)(Params...), uint64_t clusters, int cluster, uint32_t threads, size_t smem, int dev,
                            std::atomic<int> (&known)[64], cudaStream_t s, const Args&... args) {
    const int most = most_clusters(kernel, cluster, threads, smem, dev, known);
    if (most == 0) return cudaErrorCooperativeLaunchTooLarge;
    const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (err != cudaSuccess) return err;
    cudaLaunchAttribute attrs[2] = {};
    attrs[0].id = cudaLaunchAttributeCooperative;
    attrs[0].val.cooperative = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>((clusters < static_cast<uint64_t>(most) ? clusters : most) * cluster));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attrs;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

template <int CG, int BN, int TERMS, uint32_t CHUNK, bool BF16, bool A_MN, bool B_MN, class Epi>
cudaError_t launch_gemm(const Maps& maps, const Schedule& work, const Epi& epi, uint64_t tiles, int sms, cudaStream_t s) {
    using S = Shape<CG, BN, TERMS, CHUNK, BF16, Epi::kBuffer>;
    auto kernel = k_gemm<S, A_MN, B_MN, Epi>;
    // per device and cheap (a table lookup in the runtime): not remembered
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (err != cudaSuccess) return err;
    const uint64_t units = static_cast<uint64_t>(sms / CG);
    const int grid = static_cast<int>(tiles < units ? tiles : units) * CG;
    if (grid == 0) return cudaSuccess;
    return launch_clusters(kernel, grid, CG, S::kThreads, S::kSmem, s, true, maps, work, epi);
}

}  // namespace ops
}  // namespace dsm
