// C ABI of the operators around a selection in a decoding loop (see profk.h): argument checks, launch shapes, launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <mutex>

#include "logprobs.cuh"
#include "paged_attention.cuh"
#include "pages.cuh"
#include "profk.h"

using namespace profk;

namespace {

#define DEC_TRY(expr)                                                     \
    do {                                                                  \
        if ((expr) != cudaSuccess) { (void)cudaGetLastError(); return PROFK_ECUDA; } \
    } while (0)

constexpr int MAX_DEVICES = 64;
constexpr int64_t MAX_PAGE_SIZE = 1 << 24, MAX_TOKENS = 0x7FFFFF00ll;      // of a page, of a sequence

// Whether a table of `width` entries and pages of `page_size` tokens are within what the kernels count (no product wraps).
bool table_ok(int64_t width, int64_t page_size) { return page_size >= 1 && page_size <= MAX_PAGE_SIZE && width >= 1 && width <= MAX_TOKENS / page_size; }

// Whether the kernels can work with a factor of the exponents: it and its product with log2(e) are normal fp32 numbers (a
// factor of zero would make masked elements NaN, an infinite one all that equal the maximum).
bool factor_ok(double factor) {
    const float f = (float)factor;
    return f >= FLT_MIN && std::isfinite(f * LOG2E);
}
bool temperature_ok(double temperature) { return temperature > 0 && std::isfinite(temperature) && factor_ok(1.0 / temperature); }
float scale_of(double temperature) { return (float)(1.0 / temperature); }
float unscale_of(double temperature) { return (float)(1.0 / (double)scale_of(temperature)); }

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

// ---- log probabilities -----------------------------------------------------------------------

size_t lp_smem(unsigned parts, uint32_t k) {
    return LP_TEAMS * sizeof(LpTeamMemory) + 2 * (size_t)parts * ((k ? k + LP_SLACK : 0) * sizeof(uint64_t) + sizeof(LpStats) + 2 * sizeof(float));
}

// Clusters of `shares` CTAs (each with an SM to itself) that run at a time: the SMs of a cluster lie in one part of the
// chip, and not every part holds a multiple of them.
template <typename K>
int lp_clusters(K* kernel, unsigned shares, size_t smem, int sms) {
    if (shares == 1) return sms;
    static int known[MAX_DEVICES][5];                    // by log2 of the shares; the same for all builds of the kernel
    static std::mutex mutex;
    int dev = 0, log2 = 0, n = 0;
    while ((1u << log2) < shares) ++log2;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    std::lock_guard<std::mutex> lock(mutex);
    if (known[dev][log2] == 0) {
        Launch l(shares, LP_THREADS, smem, nullptr, shares);
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &l.cfg) != cudaSuccess || n < 1) { (void)cudaGetLastError(); n = std::max(1, sms / (int)shares); }
        known[dev][log2] = n;
    }
    return known[dev][log2];
}

// Teams per row.  The time of a row and part is that of its bytes at a team's share of the bandwidth plus a fixed latency
// (in bytes of that stream, 22 GB/s: 1 us is 22 KB), and rows beyond what runs at a time wait: the number of parts with the
// least of it.  The fixed part was read off calls with one row per team: 3 us without alternatives, 6 with them (most of
// it behind the stream, and hidden behind the next row's), and 2 more for parts that meet.
template <typename K>
unsigned lp_parts(K* kernel, int64_t rows, int64_t V, size_t elem, bool top, int sms) {
    const double us = 22000.0, bytes = (double)V * elem;
    unsigned best = 1;
    double best_cost = 0;
    for (unsigned parts = 1; parts <= LP_MAX_PARTS; parts *= 2) {
        if (parts > 1 && bytes / parts < 4096.0) break;
        const unsigned shares = std::max(1u, parts / LP_TEAMS);
        const double at_a_time = (double)lp_clusters(kernel, shares, lp_smem(LP_MAX_PARTS, LP_MAX_K), sms) * shares * LP_TEAMS / parts;
        const double rounds = std::ceil((double)rows / at_a_time);
        const double open = (top ? 1.5 : 0.5) * us + (parts > 1 ? (top ? 2.0 : 1.0) * us : 0.0), close = (top ? 4.5 : 2.5) * us;
        const double cost = rounds * (bytes / parts + open) + close;
        if (parts == 1 || cost < best_cost) { best = parts; best_cost = cost; }
    }
    return best;
}

template <typename T, bool ENT, bool TOPK>
int lp_launch(LpParams p, int sms, void* stream) {
    static uint64_t done = 0;
    static std::mutex mutex;
    auto* kernel = logprobs_kernel<T, ENT, TOPK>;
    DEC_TRY(prepare_kernel(kernel, lp_smem(LP_MAX_PARTS, LP_MAX_K), &done, &mutex));
    p.parts = lp_parts(kernel, p.rows, p.V, sizeof(T), TOPK, sms);
    for (p.parts_log2 = 0; (1u << p.parts_log2) < p.parts; ++p.parts_log2) {}
    const unsigned shares = std::max(1u, p.parts / LP_TEAMS);
    const int64_t most = lp_clusters(kernel, shares, lp_smem(LP_MAX_PARTS, LP_MAX_K), sms);
    const int64_t groups = std::min<int64_t>(p.parts > 1 ? p.rows : (p.rows + LP_TEAMS - 1) / LP_TEAMS, most);
    Launch l((unsigned)(groups * shares), LP_THREADS, lp_smem(p.parts, p.k), stream, shares);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, kernel, p));
    return PROFK_OK;
}

template <typename T>
int lp_forward(const T* logits, int64_t rows, int64_t V, int64_t row_stride, const int64_t* tokens, int64_t k, double temperature,
               void* stream, float* logprob, float* lse, float* lse_rest, float* entropy, float* top_logprobs, int64_t* top_tokens) {
    if (!logits || !lse || rows < 1 || rows > 0x7FFFFFFFll || V < 1 || V > 0x7FFFFFFFll || rows > (1ll << 40) / V || (rows > 1 && row_stride < V) || k < 0 ||
        k > LP_MAX_K || k > V || !temperature_ok(temperature) || (reinterpret_cast<uintptr_t>(logits) % sizeof(T)) != 0 || (k > 0) != (top_logprobs != nullptr) ||
        (k > 0) != (top_tokens != nullptr) || (tokens != nullptr) != (logprob != nullptr))
        return PROFK_EINVAL;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    LpParams p{logits, rows, row_stride, (uint32_t)V, (uint32_t)k, 1u, 0u, scale_of(temperature), unscale_of(temperature), tokens, logprob, lse, lse_rest, entropy, top_logprobs, top_tokens};
    if (entropy) return k ? lp_launch<T, true, true>(p, sms, stream) : lp_launch<T, true, false>(p, sms, stream);
    return k ? lp_launch<T, false, true>(p, sms, stream) : lp_launch<T, false, false>(p, sms, stream);
}

template <typename T>
int lp_backward(const T* logits, int64_t rows, int64_t V, int64_t row_stride, double temperature, const float* lse, const float* lse_rest, const int64_t* tokens,
                const float* grad_logprob, const float* entropy, const float* grad_entropy, const float* grad_lse, int64_t k,
                const int64_t* top_tokens, const float* grad_top, void* stream, T* grad, int64_t grad_row_stride) {
    if (!logits || !grad || !lse || rows < 1 || V < 1 || V > 0x7FFFFFFFll || rows > (1ll << 40) / V || (rows > 1 && (row_stride < V || grad_row_stride < V)) ||
        k < 0 || k > LP_MAX_K || k > V || !temperature_ok(temperature) ||
        (reinterpret_cast<uintptr_t>(logits) % sizeof(T)) != 0 || (reinterpret_cast<uintptr_t>(grad) % sizeof(T)) != 0 ||
        (grad_logprob && !tokens) || (grad_entropy && !entropy) || (grad_top && (!top_tokens || k < 1)))
        return PROFK_EINVAL;
    if (grad == logits && (grad_logprob || grad_top || (rows > 1 && grad_row_stride != row_stride))) return PROFK_EINVAL;
    const uint32_t most = LG_THREADS * LG_UNROLL * 2 * Logit<T>::VEC;
    const uint32_t chunk = (uint32_t)std::min<int64_t>(most, (V + 15) / 16 * 16);
    const int64_t chunks = (V + chunk - 1) / chunk;
    if (rows * chunks > 0x7FFFFFFFll) return PROFK_EINVAL;
    LpGradParams p{logits, grad, rows, row_stride, grad_row_stride, (uint32_t)V, grad_top ? (uint32_t)k : 0u, (uint32_t)chunks, chunk,
                   scale_of(temperature), unscale_of(temperature), tokens, lse, lse_rest, entropy, grad_logprob, grad_entropy, grad_lse, top_tokens, grad_top};
    Launch l((unsigned)(rows * chunks), LG_THREADS, 0, stream);
    const bool shifted = (reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(grad)) % 16 != 0 ||
                         (rows > 1 && (row_stride - grad_row_stride) * (int64_t)sizeof(T) % 16 != 0);
    DEC_TRY(shifted ? cudaLaunchKernelEx(&l.cfg, logprobs_grad_kernel<T, true>, p) : cudaLaunchKernelEx(&l.cfg, logprobs_grad_kernel<T, false>, p));
    return PROFK_OK;
}

// ---- paged attention -------------------------------------------------------------------------

constexpr int PA_MAX_DIM = 256;

int pa_tile_dim(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
size_t pa_meta_bytes(int sms) { return ((size_t)sms * sizeof(PaMeta) + 255) / 256 * 256; }
size_t pa_workspace(int64_t dim, int sms) {
    const int d = pa_tile_dim(dim);
    const size_t slots = d == 64 ? PaShape<64>::SLOTS : d == 128 ? PaShape<128>::SLOTS : PaShape<256>::SLOTS;
    return pa_meta_bytes(sms) + (size_t)sms * slots * PA_ROWS * (d + 2) * sizeof(float);
}
int pa_warps(int64_t dim) {
    const int d = pa_tile_dim(dim);
    return d == 64 ? PaShape<64>::WARPS : d == 128 ? PaShape<128>::WARPS : PaShape<256>::WARPS;
}

template <typename T, int D, int N8>
int pa_launch(const PaParams& p, unsigned ctas, void* stream) {
    static uint64_t done = 0;
    static std::mutex mutex;
    DEC_TRY(prepare_kernel(paged_attention_kernel<T, D, N8>, PaShape<D>::SMEM, &done, &mutex));
    Launch l(ctas, PaShape<D>::THREADS, PaShape<D>::SMEM, stream);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, paged_attention_kernel<T, D, N8>, p));
    Launch j(ctas, PJ_THREADS, 0, stream);
    j.cfg.gridDim.y = (unsigned)p.rows;
    DEC_TRY(cudaLaunchKernelEx(&j.cfg, paged_attention_join_kernel<T, D>, p));
    return PROFK_OK;
}
template <typename T, int D>
int pa_launch(const PaParams& p, unsigned ctas, void* stream) {
    return p.rows <= 8 ? pa_launch<T, D, 1>(p, ctas, stream) : pa_launch<T, D, 2>(p, ctas, stream);
}

int32_t log2_of(int64_t n) {      // -1: no power of two
    int32_t s = 0;
    while ((int64_t)1 << s < n) ++s;
    return (int64_t)1 << s == n ? s : -1;
}
// Whether a page's tokens lie within 2^32 bytes (of two-byte elements) behind the first.
bool spans_32_bits(int64_t page_size, int64_t token) { return token >= 0 && token <= (0xFFFFFFFFll / 2) / (page_size + PA_SUB); }
bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

template <typename T>
int pa_run(const T* q, int64_t q_seq, int64_t q_head, const T* k, const T* v, const profk_page_strides_t* ks, const profk_page_strides_t* vs,
           const int32_t* tables, int64_t table_stride, const int32_t* lengths, int64_t seqs, int64_t heads, int64_t kv_heads, int64_t dim,
           int64_t page_size, int64_t pages, int64_t width, double scale, void* workspace, size_t workspace_bytes, void* stream, T* out, float* lse) {
    if (!q || !k || !v || !ks || !vs || !tables || !lengths || !out || !lse || seqs < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0 ||
        dim < 8 || dim > PA_MAX_DIM || dim % 8 != 0 || !table_ok(width, page_size) || pages < 1 || seqs > (1 << 24) || heads > (1 << 16) ||
        pages > 0x7FFFFFFFll || table_stride < 0 || !factor_ok(scale) ||
        !aligned_to(q, 4) || q_seq % 2 != 0 || q_head % 2 != 0 || !aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(out, 16))
        return PROFK_EINVAL;
    for (const profk_page_strides_t* s : {ks, vs})
        if (s->page % 8 != 0 || s->head % 8 != 0 || s->token % 8 != 0) return PROFK_EINVAL;
    if ((width * page_size / PA_SUB + 1) * kv_heads * ((heads / kv_heads + PA_ROWS - 1) / PA_ROWS) > 0x7FFFFFFFll) return PROFK_EINVAL;   // tiles of a sequence
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    const size_t need = pa_workspace(dim, sms);
    if (!workspace || workspace_bytes < need || !aligned_to(workspace, 256)) return PROFK_EWORKSPACE;
    const int32_t group = (int32_t)(heads / kv_heads), blocks = (group + PA_ROWS - 1) / PA_ROWS;
    // no more warps than there can be shares, or sequences without tokens
    const int64_t tiles = seqs * kv_heads * blocks * ((width * page_size + PA_SUB - 1) / PA_SUB);
    const int64_t most = std::max<int64_t>(seqs, tiles), warps = pa_warps(dim);
    const unsigned ctas = (unsigned)std::min<int64_t>(sms, (most + warps - 1) / warps);
    PaParams p{q, k, v, q_seq, q_head, ks->page, ks->head, ks->token, vs->page, vs->head, vs->token, tables, table_stride, lengths,
               (int32_t)seqs, (int32_t)heads, (int32_t)kv_heads, group, (int32_t)dim, (int32_t)page_size, (int32_t)pages, (int32_t)width,
               blocks, (group + blocks - 1) / blocks, log2_of(page_size), page_size % PA_SUB == 0 && spans_32_bits(page_size, ks->token) && spans_32_bits(page_size, vs->token), (float)scale, out, lse,
               reinterpret_cast<float*>(static_cast<char*>(workspace) + pa_meta_bytes(sms)), static_cast<PaMeta*>(workspace)};
    switch (pa_tile_dim(dim)) {
        case 64: return pa_launch<T, 64>(p, ctas, stream);
        case 128: return pa_launch<T, 128>(p, ctas, stream);
        default: return pa_launch<T, 256>(p, ctas, stream);
    }
}

// ---- pages -----------------------------------------------------------------------------------

bool pg_pool_ok(const profk_pool_t* pool) {
    if (!pool) return true;
    return pool->base && aligned_to(pool->base, 16) && pool->layers >= 1 && pool->layers <= (1 << 20) && pool->kv_heads >= 1 && pool->kv_heads <= (1 << 16) &&
           pool->page_size >= 1 && pool->page_size <= MAX_PAGE_SIZE && pool->row_bytes >= 16 && pool->row_bytes <= (1 << 20) && pool->row_bytes % 16 == 0 && pool->layer % 16 == 0 &&
           pool->kv % 16 == 0 && pool->page % 16 == 0 && pool->head % 16 == 0 && pool->token % 16 == 0 &&
           pool->kv_heads * pool->page_size * (pool->row_bytes / 16) <= (1 << 30);
}
// `unroll`: vectors per thread that are in flight at a time; a plane is copied by as few threads as hold it so.
PgPool pg_pool(const profk_pool_t* pool, int64_t page_size, int unroll) {
    if (!pool) return PgPool{nullptr, 0, 0, (int32_t)page_size, 0, PG_THREADS, 0, 0, 0, 0, 0};
    const int64_t vectors = pool->kv_heads * pool->page_size * (pool->row_bytes / 16);
    int team = 32;
    while (team < PG_THREADS && team * unroll < vectors) team *= 2;
    return PgPool{static_cast<char*>(pool->base), (int32_t)pool->layers, (int32_t)pool->kv_heads, (int32_t)pool->page_size, (int32_t)pool->row_bytes, team,
                  pool->layer, pool->kv, pool->page, pool->head, pool->token};
}
size_t up(size_t n) { return (n + 255) / 256 * 256; }
int64_t fork_fresh(int64_t n, int64_t pages, int64_t page_size, int64_t grow) { return std::min(pages, n * (1 + (grow + page_size - 1) / page_size)); }
size_t fork_workspace(int64_t n_old, int64_t n, int64_t pages, int64_t page_size, int64_t grow) {
    return 256 + 2 * up((size_t)n_old * 4) + up((size_t)n * 4) + up((size_t)fork_fresh(n, pages, page_size, grow) * 4) + up((size_t)n * sizeof(PgMove));
}
bool fork_sizes_ok(int64_t n_old, int64_t n, int64_t pages, int64_t page_size, int64_t grow) {
    return n_old >= 0 && n >= 0 && n_old <= (1 << 24) && n <= (1 << 24) && pages >= 1 && pages <= 0x7FFF0000ll && page_size >= 1 && page_size <= MAX_PAGE_SIZE &&
           grow >= 0 && grow <= (1 << 24) && n * (1 + (grow + page_size - 1) / page_size) <= 0x7FFF0000ll;
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

int profk_paged_attention_workspace_bytes(int64_t dim, size_t* bytes) {
    if (!bytes || dim < 8 || dim > PA_MAX_DIM || dim % 8 != 0) return PROFK_EINVAL;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    *bytes = pa_workspace(dim, sms);
    return PROFK_OK;
}

#define PROFK_DEFINE_ATTENTION(SUFFIX, ELEM)                                                                                            \
    int profk_paged_attention_##SUFFIX(const void* q, int64_t q_seq_stride, int64_t q_head_stride, const void* k_pages, const void* v_pages, \
                                       const profk_page_strides_t* k_strides, const profk_page_strides_t* v_strides, const int32_t* tables, \
                                       int64_t table_stride, const int32_t* lengths, int64_t seqs, int64_t heads, int64_t kv_heads, int64_t dim, \
                                       int64_t page_size, int64_t pages, int64_t width, double scale, void* workspace,                  \
                                       size_t workspace_bytes, void* stream, void* out, float* lse) {                                   \
        return pa_run<ELEM>((const ELEM*)q, q_seq_stride, q_head_stride, (const ELEM*)k_pages, (const ELEM*)v_pages, k_strides, v_strides, tables, \
                            table_stride, lengths, seqs, heads, kv_heads, dim, page_size, pages, width, scale, workspace, workspace_bytes, \
                            stream, (ELEM*)out, lse);                                                                                   \
    }

PROFK_DEFINE_ATTENTION(bf16, __nv_bfloat16)
PROFK_DEFINE_ATTENTION(f16, __half)

int profk_pages_fork_workspace_bytes(int64_t n_old, int64_t n, int64_t pages, int64_t page_size, int64_t grow, size_t* bytes) {
    if (!bytes || !fork_sizes_ok(n_old, n, pages, page_size, grow)) return PROFK_EINVAL;
    *bytes = fork_workspace(n_old, n, pages, page_size, grow);
    return PROFK_OK;
}

int profk_pages_fork(const profk_pool_t* pool, const int32_t* tables, int64_t n_old, int64_t width, int64_t table_stride, const int32_t* lengths,
                     const int32_t* refs, int64_t pages, const int32_t* parents, int64_t n, int64_t page_size, int64_t grow, void* workspace,
                     size_t workspace_bytes, void* stream, int32_t* out_tables, int32_t* out_lengths, int32_t* out_refs, int32_t* out_missing) {
    return profk_pages_fork_ex(pool, tables, n_old, width, table_stride, lengths, refs, pages, parents, n, page_size, grow, 0, workspace, workspace_bytes, stream,
                               out_tables, out_lengths, out_refs, out_missing);
}

int profk_pages_fork_ex(const profk_pool_t* pool, const int32_t* tables, int64_t n_old, int64_t width, int64_t table_stride, const int32_t* lengths,
                        const int32_t* refs, int64_t pages, const int32_t* parents, int64_t n, int64_t page_size, int64_t grow, int flags, void* workspace,
                        size_t workspace_bytes, void* stream, int32_t* out_tables, int32_t* out_lengths, int32_t* out_refs, int32_t* out_missing) {
    if ((flags & ~PROFK_FORK_PAST_ROOM) != 0 || !fork_sizes_ok(n_old, n, pages, page_size, grow) || !table_ok(width, page_size) || table_stride < 0 || !refs || !out_refs ||
        out_refs == refs || !out_missing || (n_old > 0 && (!tables || !lengths)) || (n > 0 && (!parents || !out_tables || !out_lengths)) ||
        (n > 0 && (out_tables == tables || out_lengths == lengths)) || !pg_pool_ok(pool) || (pool && pool->page_size != page_size))
        return PROFK_EINVAL;
    if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < fork_workspace(n_old, n, pages, page_size, grow)) return PROFK_EWORKSPACE;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    char* w = static_cast<char*>(workspace);
    auto take = [&](size_t bytes) { char* at = w; w += up(bytes); return at; };
    PgForkParams p{};
    p.tables = tables;
    p.table_stride = table_stride;
    p.lengths = lengths;
    p.refs = refs;
    p.parents = parents;
    p.n_old = (int32_t)n_old;
    p.n = (int32_t)n;
    p.width = (int32_t)width;
    p.pages = (int32_t)pages;
    p.page_size = (int32_t)page_size;
    p.grow = (int32_t)grow;
    p.past_room = (flags & PROFK_FORK_PAST_ROOM) != 0;
    p.out_tables = out_tables;
    p.out_lengths = out_lengths;
    p.out_refs = out_refs;
    p.out_missing = out_missing;
    p.head = reinterpret_cast<PgPlanHead*>(take(sizeof(PgPlanHead)));
    p.first = reinterpret_cast<int32_t*>(take((size_t)n_old * 4));
    p.kids = reinterpret_cast<int32_t*>(take((size_t)n_old * 4));
    p.need = reinterpret_cast<int32_t*>(take((size_t)n * 4));
    p.fresh = reinterpret_cast<int32_t*>(take((size_t)fork_fresh(n, pages, page_size, grow) * 4));
    p.moves = reinterpret_cast<PgMove*>(take((size_t)n * sizeof(PgMove)));
    p.pool = pg_pool(pool, page_size, PG_UNROLL_PIECES);
    const unsigned copiers = (unsigned)std::min<int64_t>(sms, (pages + PG_PLAN_THREADS - 1) / PG_PLAN_THREADS);
    Launch plan(1 + copiers, PG_PLAN_THREADS, 0, stream);
    DEC_TRY(cudaLaunchKernelEx(&plan.cfg, pages_fork_plan_kernel, p));
    Launch work((unsigned)sms * PG_CTAS_PIECES, PG_THREADS, 0, stream);
    DEC_TRY(cudaLaunchKernelEx(&work.cfg, pages_fork_kernel, p));
    return PROFK_OK;
}

static size_t compact_workspace(int64_t pages) { return 256 + up((size_t)pages * 4) + up((size_t)(pages / 2 + 1) * sizeof(PgMove)); }

int profk_pages_compact_workspace_bytes(int64_t pages, size_t* bytes) {
    if (!bytes || pages < 1 || pages > 0x7FFF0000ll) return PROFK_EINVAL;
    *bytes = compact_workspace(pages);
    return PROFK_OK;
}

int profk_pages_compact(const profk_pool_t* pool, const int32_t* tables, int64_t n, int64_t width, int64_t table_stride, const int32_t* refs,
                        int64_t pages, void* workspace, size_t workspace_bytes, void* stream, int32_t* out_tables, int32_t* out_refs,
                        int32_t* out_page_map, int32_t* out_live) {
    if (n < 0 || n > (1 << 24) || width < 1 || width > 0x7FFFFF00ll || table_stride < 0 || pages < 1 || pages > 0x7FFF0000ll || !refs || !out_refs ||
        refs == out_refs || !out_page_map || !out_live || (n > 0 && (!tables || !out_tables || tables == out_tables)) || !pg_pool_ok(pool))
        return PROFK_EINVAL;
    if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < compact_workspace(pages)) return PROFK_EWORKSPACE;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    char* w = static_cast<char*>(workspace) + 256;
    const int64_t step = 4 * PG_PLAN_THREADS, steps = (pages + step - 1) / step, share = (steps + sms - 1) / sms * step;
    PgCompactParams p{tables, table_stride, refs, (int32_t)n, (int32_t)width, (int32_t)pages, out_tables, out_refs, out_page_map, out_live,
                      static_cast<PgPlanHead*>(workspace), reinterpret_cast<int32_t*>(w), (int32_t)share,
                      reinterpret_cast<PgMove*>(w + up((size_t)pages * 4)), pg_pool(pool, 1, PG_UNROLL_PAGES)};
    Launch plan((unsigned)((pages + share - 1) / share), PG_PLAN_THREADS, 0, stream);
    DEC_TRY(cudaLaunchKernelEx(&plan.cfg, pages_compact_plan_kernel, p));
    Launch work((unsigned)sms * PG_CTAS_PAGES, PG_THREADS, 0, stream);
    DEC_TRY(cudaLaunchKernelEx(&work.cfg, pages_compact_kernel, p));
    return PROFK_OK;
}

int profk_pages_copy(const profk_pool_t* pool, int64_t pages, const int32_t* src, const int32_t* dst, int64_t n, void* stream) {
    if (!pool || !pg_pool_ok(pool) || pages < 1 || pages > 0x7FFF0000ll || n < 0 || n > 0x7FFF0000ll || (n > 0 && (!src || !dst))) return PROFK_EINVAL;
    if (n == 0) return PROFK_OK;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    PgCopyParams p{src, dst, (int32_t)n, (int32_t)pages, pg_pool(pool, pool->page_size, PG_UNROLL_PAGES)};
    Launch l((unsigned)std::min<int64_t>((int64_t)sms * PG_CTAS_PAGES, n * 2 * pool->layers), PG_THREADS, 0, stream);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, pages_copy_kernel, p));
    return PROFK_OK;
}

int profk_pages_append(const void* k, const void* v, const int64_t* k_strides, const int64_t* v_strides, void* k_pages, void* v_pages,
                       const profk_page_strides_t* kp, const profk_page_strides_t* vp, const int32_t* tables, int64_t table_stride,
                       const int32_t* lengths, int64_t seqs, int64_t tokens, int64_t kv_heads, int64_t row_bytes, int64_t page_size,
                       int64_t pages, int64_t width, void* stream) {
    if (!k || !v || !k_strides || !v_strides || !k_pages || !v_pages || !kp || !vp || !tables || !lengths || seqs < 1 || seqs > (1 << 24) || tokens < 1 ||
        kv_heads < 1 || kv_heads > (1 << 16) || row_bytes < 16 || row_bytes > (1 << 20) || row_bytes % 16 != 0 || !table_ok(width, page_size) || pages < 1 ||
        pages > 0x7FFFFFFFll || tokens > width * page_size || table_stride < 0 || !aligned_to(k, 16) ||
        !aligned_to(v, 16) || !aligned_to(k_pages, 16) || !aligned_to(v_pages, 16))
        return PROFK_EINVAL;
    for (const int64_t x : {k_strides[0], k_strides[1], k_strides[2], v_strides[0], v_strides[1], v_strides[2], kp->page, kp->head, kp->token, vp->page,
                            vp->head, vp->token})
        if (x % 16 != 0) return PROFK_EINVAL;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    PgAppendParams p{static_cast<const char*>(k), static_cast<const char*>(v), k_strides[0], k_strides[1], k_strides[2], v_strides[0], v_strides[1],
                     v_strides[2], static_cast<char*>(k_pages), static_cast<char*>(v_pages), kp->page, kp->head, kp->token, vp->page, vp->head, vp->token,
                     tables, table_stride, lengths, (int32_t)seqs, (int32_t)tokens, (int32_t)kv_heads, (int32_t)row_bytes, (int32_t)page_size,
                     (int32_t)pages, (int32_t)width};
    const int64_t n = seqs * tokens * kv_heads * (row_bytes / 16);
    Launch l((unsigned)std::min<int64_t>((int64_t)sms * 8, (n + PG_THREADS - 1) / PG_THREADS), PG_THREADS, 0, stream);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, pages_append_kernel, p));
    return PROFK_OK;
}

}  // extern "C"
