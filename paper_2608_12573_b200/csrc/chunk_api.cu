// C ABI of the attention of a chunk of new tokens over a paged cache (see profk.h): argument checks, launch shapes, launches.
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <numeric>
#include <type_traits>

#include "chunk_attention.cuh"
#include "decode_host.cuh"

using namespace profk;

namespace {

constexpr int CA_MAX_DIM = 256;
constexpr unsigned CA_JOIN_ROWS = 8;                    // CTAs that share the rows of an item
std::atomic<int32_t> g_polls{CA_POLLS};                 // see profk_debug_set_chunk_wait_polls

int ca_tile_dim(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
size_t ca_round(size_t n) { return (n + 255) / 256 * 256; }
size_t ca_meta_bytes(int sms) { return ca_round((size_t)sms * 2 * sizeof(CaMeta)); }
size_t ca_sums_bytes(int sms, int block) { return ca_round((size_t)sms * 2 * block * sizeof(float2)); }
int ca_block(int d) { return d == 256 ? CaShape<256>::BLOCK : CaShape<128>::BLOCK; }
size_t ca_workspace(int64_t dim, int sms) {
    const int d = ca_tile_dim(dim), block = ca_block(d);
    return ca_meta_bytes(sms) + ca_sums_bytes(sms, block) + (size_t)sms * 2 * block * d * sizeof(float);
}

// Registers: the launch's share must cover what the warpgroups ask for afterwards, or they would wait for good.
template <typename K>
cudaError_t ca_prepare(K* kernel, size_t smem, uint64_t* done, std::mutex* mutex) {
    cudaFuncAttributes a;
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    {
        std::lock_guard<std::mutex> lock(*mutex);
        if (*done >> dev & 1) return cudaSuccess;
    }
    if ((err = cudaFuncGetAttributes(&a, kernel)) != cudaSuccess) return err;
    if (a.numRegs * CA_THREADS < CA_MANY_REGISTERS * 256 + CA_FEW_REGISTERS * (CA_THREADS - 256)) return cudaErrorInvalidConfiguration;
    return prepare_kernel(kernel, smem, done, mutex);
}

// The driver's function that writes a tensor map; null: not to be had.
PFN_cuTensorMapEncodeTiled_v12000 ca_encoder() {
    static const auto encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
    }();
    return encode;
}

// Four dimensions (the first dense), strides of the others in elements; boxes of 64 elements x `second` x `third` x 1, swizzled.
// False where such copies cannot be had (a stride of zero, or too long a one).
template <typename T>
bool ca_map(CUtensorMap* map, const T* base, const int64_t* sizes, const int64_t* steps, int64_t second, int64_t third) {
    const auto encode = ca_encoder();
    if (!encode || second > 256 || third > 256) return false;
    cuuint64_t dims[4], strides[3];
    for (int i = 0; i < 4; ++i) dims[i] = (cuuint64_t)sizes[i];
    for (int i = 0; i < 3; ++i) {
        const int64_t step = sizes[i + 1] == 1 ? (sizes[0] + 7) / 8 * 8 : steps[i];        // (of one there is no stride)
        if (step <= 0 || step % 8 != 0 || step >= (1ll << 40) / (int64_t)sizeof(T)) return false;
        strides[i] = (cuuint64_t)step * sizeof(T);
    }
    const cuuint32_t box[4] = {64, (cuuint32_t)second, (cuuint32_t)third, 1}, ones[4] = {1, 1, 1, 1};
    const CUtensorMapDataType type = std::is_same_v<T, __half> ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return encode(map, type, 4, const_cast<T*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D>
int ca_launch(CaParams<T> p, const CaMaps& maps, int sms, void* workspace, void* stream) {
    static uint64_t done = 0;
    static std::mutex mutex;
    DEC_TRY(ca_prepare(paged_attention_chunk_kernel<T, D>, ca_smem_bytes<D>(), &done, &mutex));
    char* w = static_cast<char*>(workspace);
    p.meta = reinterpret_cast<CaMeta*>(w);
    p.sums = reinterpret_cast<float2*>(w + ca_meta_bytes(sms));
    p.parts = reinterpret_cast<float*>(w + ca_meta_bytes(sms) + ca_sums_bytes(sms, CaShape<D>::BLOCK));
    Launch l((unsigned)sms, CA_THREADS, ca_smem_bytes<D>(), stream);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, paged_attention_chunk_kernel<T, D>, p, maps));
    Launch j((unsigned)sms, CJ_THREADS, 0, stream);
    j.cfg.gridDim.y = CA_JOIN_ROWS;
    DEC_TRY(cudaLaunchKernelEx(&j.cfg, paged_attention_chunk_join_kernel<T, D>, p, (int32_t)sms));
    return PROFK_OK;
}

template <typename T>
int ca_run(const T* q, const int64_t* qs, const T* k, const T* v, const profk_page_strides_t* ks, const profk_page_strides_t* vs, const int32_t* tables,
           int64_t table_stride, const int32_t* lengths, const int32_t* starts, int64_t seqs, int64_t rows, int64_t heads, int64_t kv_heads, int64_t dim,
           int64_t page_size, int64_t pages, int64_t width, double scale, void* workspace, size_t workspace_bytes, void* stream, T* out, float* lse) {
    if (!q || !qs || !k || !v || !ks || !vs || !tables || !lengths || !out || !lse || seqs < 1 || seqs > (1 << 24) || rows < 1 || heads < 1 || heads > (1 << 16) ||
        kv_heads < 1 || heads % kv_heads != 0 || rows > 0x7FFFFFFFll / heads || (!starts && rows % seqs != 0) || dim < 8 || dim > CA_MAX_DIM || dim % 8 != 0 ||
        !table_ok(width, page_size) || pages < 1 || pages > 0x7FFFFFFFll || table_stride < 0 || !factor_ok(scale) || !aligned_to(q, sizeof(T)) || !aligned_to(k, 16) ||
        !aligned_to(v, 16) || !aligned_to(out, 16))
        return PROFK_EINVAL;
    for (const profk_page_strides_t* s : {ks, vs})
        if (s->page % 8 != 0 || s->head % 8 != 0 || s->token % 8 != 0) return PROFK_EINVAL;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    if (!workspace || workspace_bytes < ca_workspace(dim, sms) || !aligned_to(workspace, 256)) return PROFK_EWORKSPACE;
    CaParams<T> p{};
    p.q = q;
    p.q_seq = qs[0];
    p.q_token = qs[1];
    p.q_head = qs[2];
    p.q_wide = aligned_to(q, 16) && qs[0] % 8 == 0 && qs[1] % 8 == 0 && qs[2] % 8 == 0;
    p.k = k;
    p.v = v;
    p.ks_page = ks->page;
    p.ks_head = ks->head;
    p.ks_token = ks->token;
    p.vs_page = vs->page;
    p.vs_head = vs->head;
    p.vs_token = vs->token;
    p.tables = tables;
    p.table_stride = table_stride;
    p.lengths = lengths;
    p.starts = starts;
    p.rows = rows;
    p.tokens = starts ? 0 : rows / seqs;
    p.seqs = (int32_t)seqs;
    p.heads = (int32_t)heads;
    p.kv_heads = (int32_t)kv_heads;
    p.group = (int32_t)(heads / kv_heads);
    p.dim = (int32_t)dim;
    p.page_size = (int32_t)page_size;
    p.pages = (int32_t)pages;
    p.width = (int32_t)width;
    p.by_group = CaDivisor::of((uint32_t)p.group);
    p.by_page = CaDivisor::of((uint32_t)page_size);
    p.scale = (float)scale;
    p.polls = g_polls.load(std::memory_order_relaxed);
    p.out = out;
    p.lse = lse;
    // copies by tile want boxes of eight tokens (one atom of the swizzle) at least that never leave a page
    CaMaps maps{};
    const int tile_dim = ca_tile_dim(dim), tile = tile_dim == 256 ? CaShape<256>::KT : CaShape<128>::KT;
    const int box = (int)std::gcd(page_size, (int64_t)tile);
    const int64_t kv_sizes[4] = {dim, page_size, kv_heads, pages}, k_steps[3] = {ks->token, ks->head, ks->page}, v_steps[3] = {vs->token, vs->head, vs->page};
    if (box >= 8 && ca_map<T>(&maps.k, k, kv_sizes, k_steps, box, 1) && ca_map<T>(&maps.v, v, kv_sizes, v_steps, box, 1)) p.box = box;
    if (p.box && p.q_wide && CA_ROWS % p.group == 0) {
        const int64_t sizes[4] = {dim, heads, starts ? rows : p.tokens, starts ? 1 : seqs}, steps[3] = {qs[2], qs[1], qs[0]};
        p.q_box = ca_map<T>(&maps.q, q, sizes, steps, p.group, CA_ROWS / p.group);
    }
    switch (tile_dim) {
        case 64: return ca_launch<T, 64>(p, maps, sms, workspace, stream);
        case 128: return ca_launch<T, 128>(p, maps, sms, workspace, stream);
        default: return ca_launch<T, 256>(p, maps, sms, workspace, stream);
    }
}

}  // namespace

extern "C" {

int profk_paged_attention_chunk_workspace_bytes(int64_t dim, size_t* bytes) {
    if (!bytes || dim < 8 || dim > CA_MAX_DIM || dim % 8 != 0) return PROFK_EINVAL;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    *bytes = ca_workspace(dim, sms);
    return PROFK_OK;
}

int profk_debug_set_chunk_wait_polls(int64_t polls) {
    g_polls.store(polls < 0 ? CA_POLLS : (int32_t)std::min<int64_t>(polls, CA_POLLS), std::memory_order_relaxed);
    return PROFK_OK;
}

#define PROFK_DEFINE_CHUNK(SUFFIX, ELEM)                                                                                                             \
    int profk_paged_attention_chunk_##SUFFIX(const void* q, const int64_t* q_strides, const void* k_pages, const void* v_pages,                      \
                                             const profk_page_strides_t* k_strides, const profk_page_strides_t* v_strides, const int32_t* tables,    \
                                             int64_t table_stride, const int32_t* lengths, const int32_t* starts, int64_t seqs, int64_t rows,        \
                                             int64_t heads, int64_t kv_heads, int64_t dim, int64_t page_size, int64_t pages, int64_t width,          \
                                             double scale, void* workspace, size_t workspace_bytes, void* stream, void* out, float* lse) {           \
        return ca_run<ELEM>((const ELEM*)q, q_strides, (const ELEM*)k_pages, (const ELEM*)v_pages, k_strides, v_strides, tables, table_stride,       \
                            lengths, starts, seqs, rows, heads, kv_heads, dim, page_size, pages, width, scale, workspace, workspace_bytes, stream,   \
                            (ELEM*)out, lse);                                                                                                        \
    }

PROFK_DEFINE_CHUNK(bf16, __nv_bfloat16)
PROFK_DEFINE_CHUNK(f16, __half)

}  // extern "C"
