// C ABI of the operators around a selection in a decoding loop (see profk.h): argument checks, launch shapes, launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>

#include "logprobs.cuh"
#include "profk.h"

using namespace profk;

namespace {

#define DEC_TRY(expr)                                                     \
    do {                                                                  \
        if ((expr) != cudaSuccess) { (void)cudaGetLastError(); return PROFK_ECUDA; } \
    } while (0)

constexpr int MAX_DEVICES = 64;

// Streaming multiprocessors of the current device; 0 on an error.
int sm_count() {
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

// Allows `kernel` its dynamic shared memory (and clusters beyond 8 CTAs where asked) once per device.
template <typename K>
cudaError_t prepare_kernel(K* kernel, size_t smem, bool wide_cluster, uint64_t* done_mask, std::mutex* mutex) {
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    std::lock_guard<std::mutex> lock(*mutex);
    if (*done_mask >> dev & 1) return cudaSuccess;
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err == cudaSuccess && wide_cluster) err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
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

// ---- log probabilities -----------------------------------------------------------------------

constexpr unsigned LP_MAX_PARTS = 16;

size_t lp_smem(unsigned parts, uint32_t k) {
    size_t bytes = (size_t)LP_STAGES * LP_UNROLL * LP_THREADS * 16;
    if (parts > 1) bytes += 2 * (size_t)parts * ((k ? k + LP_SLACK : 0) * sizeof(uint64_t) + sizeof(LpStats));
    return bytes;
}

// CTAs per row: as many as keep the device's two CTAs per SM evenly loaded, with a fixed cost per row and part that is
// the time of about a quarter of a million bytes divided among the parts.
unsigned lp_parts(int64_t rows, int64_t V, size_t elem, int sms) {
    const double slots = 2.0 * sms, fixed = 16384.0, bytes = (double)V * elem;
    unsigned best = 1;
    double best_cost = 0;
    for (unsigned parts = 1; parts <= LP_MAX_PARTS; parts *= 2) {
        if (parts > 1 && bytes / parts < 8192.0) break;
        const double rounds = std::ceil((double)rows * parts / slots);
        const double cost = rounds * (bytes / parts + fixed + (parts > 1 ? fixed : 0.0));
        if (parts == 1 || cost < best_cost) { best = parts; best_cost = cost; }
    }
    return best;
}

template <typename T, bool ENT, bool TOPK>
int lp_launch(const LpParams& p, unsigned parts, int sms, void* stream) {
    static uint64_t done = 0;
    static std::mutex mutex;
    DEC_TRY(prepare_kernel(logprobs_kernel<T, ENT, TOPK>, lp_smem(LP_MAX_PARTS, LP_MAX_K), true, &done, &mutex));
    const int64_t clusters = std::min<int64_t>(p.rows, std::max<int64_t>(1, 2 * (int64_t)sms / parts));
    Launch l((unsigned)(clusters * parts), LP_THREADS, lp_smem(parts, p.k), stream, parts);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, logprobs_kernel<T, ENT, TOPK>, p));
    return PROFK_OK;
}

template <typename T>
int lp_forward(const T* logits, int64_t rows, int64_t V, int64_t row_stride, const int64_t* tokens, int64_t k, double temperature,
               void* stream, float* logprob, float* lse, float* lse_rest, float* entropy, float* top_logprobs, int64_t* top_tokens) {
    if (!logits || !lse || rows < 1 || V < 1 || V > 0x7FFFFFFFll || rows > (1ll << 40) / V || (rows > 1 && row_stride < V) || k < 0 ||
        k > LP_MAX_K || k > V || !(temperature > 0) || !std::isfinite(temperature) || !std::isfinite(1.0 / temperature) ||
        (reinterpret_cast<uintptr_t>(logits) % sizeof(T)) != 0 || (k > 0) != (top_logprobs != nullptr) ||
        (k > 0) != (top_tokens != nullptr) || (tokens != nullptr) != (logprob != nullptr))
        return PROFK_EINVAL;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    LpParams p{logits, rows, row_stride, (uint32_t)V, (uint32_t)k, (float)(1.0 / temperature), tokens, logprob, lse, lse_rest, entropy, top_logprobs, top_tokens};
    const unsigned parts = lp_parts(rows, V, sizeof(T), sms);
    if (entropy) return k ? lp_launch<T, true, true>(p, parts, sms, stream) : lp_launch<T, true, false>(p, parts, sms, stream);
    return k ? lp_launch<T, false, true>(p, parts, sms, stream) : lp_launch<T, false, false>(p, parts, sms, stream);
}

template <typename T>
int lp_backward(const T* logits, int64_t rows, int64_t V, int64_t row_stride, double temperature, const float* lse, const float* lse_rest, const int64_t* tokens,
                const float* grad_logprob, const float* entropy, const float* grad_entropy, const float* grad_lse, int64_t k,
                const int64_t* top_tokens, const float* grad_top, void* stream, T* grad, int64_t grad_row_stride) {
    if (!logits || !grad || !lse || rows < 1 || V < 1 || V > 0x7FFFFFFFll || rows > (1ll << 40) / V || (rows > 1 && (row_stride < V || grad_row_stride < V)) ||
        k < 0 || k > LP_MAX_K || k > V || !(temperature > 0) || !std::isfinite(temperature) || !std::isfinite(1.0 / temperature) ||
        (reinterpret_cast<uintptr_t>(logits) % sizeof(T)) != 0 || (reinterpret_cast<uintptr_t>(grad) % sizeof(T)) != 0 ||
        (grad_logprob && !tokens) || (grad_entropy && !entropy) || (grad_top && (!top_tokens || k < 1)))
        return PROFK_EINVAL;
    const uint32_t most = LG_THREADS * LG_UNROLL * 2 * Logit<T>::VEC;
    const uint32_t chunk = (uint32_t)std::min<int64_t>(most, (V + 15) / 16 * 16);
    const int64_t chunks = (V + chunk - 1) / chunk;
    if (rows * chunks > 0x7FFFFFFFll) return PROFK_EINVAL;
    LpGradParams p{logits, grad, rows, row_stride, grad_row_stride, (uint32_t)V, grad_top ? (uint32_t)k : 0u, (uint32_t)chunks, chunk,
                   (float)(1.0 / temperature), tokens, lse, lse_rest, entropy, grad_logprob, grad_entropy, grad_lse, top_tokens, grad_top};
    Launch l((unsigned)(rows * chunks), LG_THREADS, 0, stream);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, logprobs_grad_kernel<T>, p));
    return PROFK_OK;
}

}  // namespace

extern "C" {

#define PROFK_DEFINE_LOGPROBS(SUFFIX, ELEM, CTYPE)                                                                                      \
    int profk_logprobs_##SUFFIX(const CTYPE* logits, int64_t rows, int64_t V, int64_t row_stride, const int64_t* tokens, int64_t k,    \
                                double temperature, void* stream, float* logprob, float* lse, float* lse_rest, float* entropy, float* top_logprobs, \
                                int64_t* top_tokens) {                                                                                  \
        return lp_forward<ELEM>((const ELEM*)logits, rows, V, row_stride, tokens, k, temperature, stream, logprob, lse, lse_rest, entropy,  \
                                top_logprobs, top_tokens);                                                                              \
    }                                                                                                                                   \
    int profk_logprobs_backward_##SUFFIX(const CTYPE* logits, int64_t rows, int64_t V, int64_t row_stride, double temperature,          \
                                         const float* lse, const float* lse_rest, const int64_t* tokens, const float* grad_logprob, const float* entropy,      \
                                         const float* grad_entropy, const float* grad_lse, int64_t k, const int64_t* top_tokens,        \
                                         const float* grad_top, void* stream, CTYPE* grad_logits, int64_t grad_row_stride) {            \
        return lp_backward<ELEM>((const ELEM*)logits, rows, V, row_stride, temperature, lse, lse_rest, tokens, grad_logprob, entropy,             \
                                 grad_entropy, grad_lse, k, top_tokens, grad_top, stream, (ELEM*)grad_logits, grad_row_stride);         \
    }

PROFK_DEFINE_LOGPROBS(f32, float, float)
PROFK_DEFINE_LOGPROBS(bf16, __nv_bfloat16, void)
PROFK_DEFINE_LOGPROBS(f16, __half, void)

}  // extern "C"
