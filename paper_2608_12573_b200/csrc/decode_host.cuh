// Host-side helpers that the decoding operators' entry points share: limits, launch configuration, per-device facts.
#pragma once

#include <cuda_runtime.h>

#include <cfloat>
#include <cmath>
#include <mutex>

#include "logits.cuh"
#include "profk.h"

namespace profk {

#define DEC_TRY(expr)                                                     \
    do {                                                                  \
        if ((expr) != cudaSuccess) { (void)cudaGetLastError(); return PROFK_ECUDA; } \
    } while (0)

constexpr int MAX_DEVICES = 64;
constexpr int64_t MAX_PAGE_SIZE = 1 << 24, MAX_TOKENS = 0x7FFFFF00ll;      // of a page, of a sequence

// Whether a table of `width` entries and pages of `page_size` tokens are within what the kernels count (no product wraps).
inline bool table_ok(int64_t width, int64_t page_size) { return page_size >= 1 && page_size <= MAX_PAGE_SIZE && width >= 1 && width <= MAX_TOKENS / page_size; }

// Whether the kernels can work with a factor of the exponents: it and its product with log2(e) are normal fp32 numbers (a
// factor of zero would make masked elements NaN, an infinite one all that equal the maximum).
inline bool factor_ok(double factor) {
    const float f = (float)factor;
    return f >= FLT_MIN && std::isfinite(f * LOG2E);
}

// Streaming multiprocessors of the current device; 0 on an error.
inline int sm_count() {
    static int counts[MAX_DEVICES];
    static std::mutex mutex;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) { (void)cudaGetLastError(); return 0; }
    std::lock_guard<std::mutex> lock(mutex);
    if (counts[dev] == 0 && cudaDeviceGetAttribute(&counts[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    return counts[dev];
}

// Allows `kernel` its dynamic shared memory once per device.
template <typename K>
cudaError_t prepare_kernel(K* kernel, size_t smem, uint64_t* done_mask, std::mutex* mutex) {
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    std::lock_guard<std::mutex> lock(*mutex);
    if (*done_mask >> dev & 1) return cudaSuccess;
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    // all of the SM's memory as shared memory: its one CTA takes most of it
    if (err == cudaSuccess) err = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (err == cudaSuccess) *done_mask |= 1ull << dev;
    return err;
}

struct Launch {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attrs[2];
    Launch(unsigned grid, unsigned block, size_t smem, void* stream, unsigned cluster = 1) {
        cfg.gridDim = dim3(grid);
        cfg.blockDim = dim3(block);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = (cudaStream_t)stream;
        attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attrs[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attrs;
        cfg.numAttrs = 1;
        if (cluster > 1) {
            attrs[1].id = cudaLaunchAttributeClusterDimension;
            attrs[1].val.clusterDim.x = cluster;
            attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
            cfg.numAttrs = 2;
        }
    }
};

inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace profk
