// C ABI of the operators that take prompts and drafts into a decoding loop (see profk.h): rotary positions, appending with
// them, and what is laid over logits.  Argument checks, launch shapes, launches.
#include <algorithm>

#include "adjust.cuh"
#include "decode_host.cuh"
#include "rotary.cuh"

using namespace profk;

namespace {

// ---- rotary positions ------------------------------------------------------------------------

constexpr int64_t RO_MAX_DIM = 1024, RO_MAX_HEADS = 1 << 16;

bool ro_how_ok(const profk_rotary_t* how, int64_t dim) {
    return how && how->frequencies && how->pairs >= 1 && how->pairs <= RO_MAX_PAIRS && 2 * how->pairs <= dim && dim <= RO_MAX_DIM &&
           std::isfinite((float)how->magnitude);
}

// Whether everything lies on 16-byte vectors: pointers, strides (in elements) and the parts of a head.
template <typename T>
bool ro_wide(const RoParams<T>& p, bool interleaved) {
    const int64_t vec = 16 / (int64_t)sizeof(T);
    if (p.dim % vec != 0 || (interleaved ? 2 * p.pairs : p.pairs) % vec != 0) return false;
    const RoRows<const T>* rows[] = {&p.q, &p.k, &p.v};
    for (const auto* r : rows)
        if (!aligned_to(r->p, 16) || r->outer % vec != 0 || r->inner % vec != 0 || r->head % vec != 0) return false;
    const int64_t strides[] = {p.kp_page, p.kp_head, p.kp_token, p.vp_page, p.vp_head, p.vp_token};
    for (const int64_t s : strides)
        if (s % vec != 0) return false;
    return aligned_to(p.out, 16) && aligned_to(p.k_pages, 16) && aligned_to(p.v_pages, 16);
}

template <typename T, int VEC, bool INTER>
int ro_launch(RoParams<T> p, int sms, void* stream) {
    const int64_t chunks = ro_chunks<VEC, INTER>(p.dim, p.pairs), heads = p.heads + 2 * p.kv_heads;
    // four heads to a thread once that still fills the device, and tokens for four turns of a CTA's threads
    const bool many = p.rows * heads * chunks >= (int64_t)sms * RO_THREADS * 8;
    const int64_t per_token = (many ? (heads + 3) / 4 : heads) * chunks;
    const int64_t angles = RO_ANGLES / p.pairs;              // tokens whose angles a CTA has room for
    p.tokens_per_cta = (int32_t)std::clamp<int64_t>(std::min({(4 * RO_THREADS + per_token - 1) / per_token, p.rows / (4 * sms), angles}), 1, RO_TOKENS);
    const int64_t ctas = (p.rows + p.tokens_per_cta - 1) / p.tokens_per_cta;
    if (ctas > 0x7FFFFFFFll) return PROFK_EINVAL;
    Launch l((unsigned)ctas, RO_THREADS, (size_t)p.tokens_per_cta * p.pairs * sizeof(float2), stream);
    DEC_TRY(many ? cudaLaunchKernelEx(&l.cfg, rotary_kernel<T, VEC, INTER, 4>, p) : cudaLaunchKernelEx(&l.cfg, rotary_kernel<T, VEC, INTER, 1>, p));
    return PROFK_OK;
}

template <typename T>
int ro_run(RoParams<T> p, const profk_rotary_t* how, void* stream) {
    p.frequencies = how->frequencies;
    p.pairs = (int32_t)how->pairs;
    p.magnitude = (float)how->magnitude;
    p.inverse = how->inverse != 0;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    constexpr int VEC = Logit<T>::VEC;
    const bool inter = how->interleaved != 0;
    if (ro_wide(p, inter)) return inter ? ro_launch<T, VEC, true>(p, sms, stream) : ro_launch<T, VEC, false>(p, sms, stream);
    return inter ? ro_launch<T, 1, true>(p, sms, stream) : ro_launch<T, 1, false>(p, sms, stream);
}

template <typename T>
int rotary(const T* x, int64_t outer, int64_t inner, int64_t heads, int64_t dim, const int64_t* strides, const int64_t* positions, const int64_t* position_strides,
           const profk_rotary_t* how, void* stream, T* out) {
    if (!x || !out || !strides || !positions || !position_strides || outer < 1 || inner < 1 || heads < 1 || heads > RO_MAX_HEADS || !ro_how_ok(how, dim) ||
        outer > (1ll << 40) / inner || outer * inner > (1ll << 40) / (heads * dim) || !aligned_to(x, sizeof(T)) || !aligned_to(out, sizeof(T)))
        return PROFK_EINVAL;
    RoParams<T> p{};
    p.q = {x, strides[0], strides[1], strides[2]};
    p.out = out;
    p.rows = outer * inner;
    p.inner = inner;
    p.heads = (int32_t)heads;
    p.dim = (int32_t)dim;
    p.positions = positions;
    p.pos_outer = position_strides[0];
    p.pos_inner = position_strides[1];
    p.seqs = p.page_size = p.width = 1;
    return ro_run(p, how, stream);
}

template <typename T>
int append_rotary(const T* q, const int64_t* q_strides, const T* k, const int64_t* k_strides, const T* v, const int64_t* v_strides, T* k_pages, T* v_pages,
                  const profk_page_strides_t* kp, const profk_page_strides_t* vp, const int32_t* tables, int64_t table_stride, const int32_t* lengths,
                  const int32_t* starts, int64_t seqs, int64_t rows, int64_t heads, int64_t kv_heads, int64_t dim, int64_t page_size, int64_t pages, int64_t width,
                  const int64_t* positions, const int64_t* position_strides, const profk_rotary_t* how, void* stream, T* out_q) {
    if (!k || !v || !k_strides || !v_strides || !k_pages || !v_pages || !kp || !vp || !tables || !lengths || seqs < 1 || seqs > (1 << 24) || rows < 1 ||
        rows > 0x7FFFFFFFll || kv_heads < 1 || kv_heads > RO_MAX_HEADS || heads < 0 || heads > RO_MAX_HEADS || (heads > 0) != (q != nullptr) ||
        (heads > 0) != (out_q != nullptr) || (heads > 0 && !q_strides) || !ro_how_ok(how, dim) || !table_ok(width, page_size) || pages < 1 || pages > 0x7FFFFFFFll ||
        table_stride < 0 || (positions && !position_strides) || (!starts && rows % seqs != 0))
        return PROFK_EINVAL;
    for (const void* a : {(const void*)q, (const void*)out_q, (const void*)k, (const void*)v, (const void*)k_pages, (const void*)v_pages})
        if (!aligned_to(a, sizeof(T))) return PROFK_EINVAL;
    RoParams<T> p{};
    if (heads > 0) p.q = {q, q_strides[0], q_strides[1], q_strides[2]};
    p.out = out_q;
    p.rows = rows;
    p.inner = starts ? rows : rows / seqs;
    p.heads = (int32_t)heads;
    p.dim = (int32_t)dim;
    p.positions = positions;
    if (positions) {
        p.pos_outer = position_strides[0];
        p.pos_inner = position_strides[1];
    }
    p.k = {k, k_strides[0], k_strides[1], k_strides[2]};
    p.v = {v, v_strides[0], v_strides[1], v_strides[2]};
    p.kv_heads = (int32_t)kv_heads;
    p.seqs = (int32_t)seqs;
    p.page_size = (int32_t)page_size;
    p.pages = (int32_t)pages;
    p.width = (int32_t)width;
    p.k_pages = k_pages;
    p.v_pages = v_pages;
    p.kp_page = kp->page;
    p.kp_head = kp->head;
    p.kp_token = kp->token;
    p.vp_page = vp->page;
    p.vp_head = vp->head;
    p.vp_token = vp->token;
    p.tables = tables;
    p.table_stride = table_stride;
    p.lengths = lengths;
    p.starts = starts;
    return ro_run(p, how, stream);
}

// ---- penalties, biases and masks --------------------------------------------------------------

// Slices of `most` tokens; fewer rows than fill the device are cut finer, down to `least`.
template <typename T>
int ad_slice(AdParams<T>& p, int64_t tokens, uint32_t most, uint32_t least, int64_t ctas) {
    p.slice = most;
    while (p.slice / 2 >= least && p.rows * ((tokens + p.slice - 1) / p.slice) < ctas) p.slice /= 2;
    p.slices = (uint32_t)((tokens + p.slice - 1) / p.slice);
    return p.rows * p.slices > 0x7FFFFFFFll ? PROFK_EINVAL : PROFK_OK;
}

template <typename T, int BITS>
int ad_named(AdParams<T> p, int sms, void* stream) {
    static uint64_t done = 0;
    static std::mutex mutex;
    using Counters = AdCounters<BITS>;
    DEC_TRY(prepare_kernel(adjust_named_kernel<T, BITS>, Counters::bytes(Counters::SLICE) + Counters::SLICE * sizeof(uint16_t) + AD_MAX_BIASES * sizeof(AdBias), &done, &mutex));
    if (!p.tokens) {                                        // no counters: one CTA has a whole row
        p.slice = p.V;
        p.slices = 1;
    } else if (ad_slice(p, p.V, Counters::SLICE, 2048, 2 * sms) != PROFK_OK) {
        return PROFK_EINVAL;
    }
    const size_t named = p.tokens ? std::min<size_t>(p.slice, (size_t)p.history) : 0;
    Launch l((unsigned)(p.rows * p.slices), AD_NAMED_THREADS, (p.tokens ? Counters::bytes(p.slice) : 0) + p.biases * sizeof(AdBias) + named * sizeof(uint16_t), stream);
    DEC_TRY(cudaLaunchKernelEx(&l.cfg, adjust_named_kernel<T, BITS>, p));
    return PROFK_OK;
}

template <typename T>
int adjust(const T* logits, int64_t rows, int64_t V, int64_t row_stride, const profk_adjust_t* how, void* stream, T* out, int64_t out_row_stride) {
    if (!logits || !out || !how || rows < 1 || rows > (1 << 27) || V < 1 || V > 0x7FFFFF00ll || rows > (1ll << 40) / V ||
        (rows > 1 && (row_stride < V || out_row_stride < V)) || !aligned_to(logits, sizeof(T)) || !aligned_to(out, sizeof(T)) ||
        (out == logits && rows > 1 && row_stride != out_row_stride))
        return PROFK_EINVAL;
    const bool history = how->history > 0, biased = how->biases > 0;
    if (how->history < 0 || how->history >= (1 << 30) || (history && !how->tokens) || how->biases < 0 || how->biases > AD_MAX_BIASES ||
        (biased && (!how->bias_tokens || !how->bias_values)))
        return PROFK_EINVAL;
    const float rho = (float)how->repetition_value;
    if (history && ((!how->repetition && !(rho > 0.0f && std::isfinite(rho))) || (!how->frequency && !std::isfinite((float)how->frequency_value)) ||
                    (!how->presence && !std::isfinite((float)how->presence_value))))
        return PROFK_EINVAL;
    const int sms = sm_count();
    if (sms < 1) return PROFK_ECUDA;
    constexpr int64_t VEC = Logit<T>::VEC;
    AdParams<T> p{logits, out, rows, row_stride, out_row_stride, (uint32_t)V, 0, 1, history ? how->tokens : nullptr, how->history, how->token_stride, how->lengths,
                  how->prompts, how->repetition, how->frequency, how->presence, rho, (float)how->frequency_value, (float)how->presence_value,
                  biased ? how->bias_tokens : nullptr, how->bias_values, (int32_t)how->biases, how->bias_token_stride, how->bias_value_stride, how->mask,
                  how->mask_stride, false};
    if (how->mask || out != logits) {
        const int64_t slots = V + VEC - 1;                   // (the row may begin inside a vector)
        if (ad_slice(p, slots, AD_THREADS * VEC * AD_UNROLL, AD_THREADS * VEC, 2 * sms) != PROFK_OK) return PROFK_EINVAL;
        Launch l((unsigned)(p.rows * p.slices), AD_THREADS, 0, stream);
        DEC_TRY(cudaLaunchKernelEx(&l.cfg, adjust_stream_kernel<T>, p));
        p.behind_stream = true;
    }
    if (!history && !biased) return PROFK_OK;
    return how->history < AD_NARROW ? ad_named<T, 16>(p, sms, stream) : ad_named<T, 32>(p, sms, stream);
}

}  // namespace

extern "C" {

#define PROFK_DEFINE_PROMPT(SUFFIX, ELEM)                                                                                                              \
    int profk_rotary_##SUFFIX(const void* x, int64_t outer, int64_t inner, int64_t heads, int64_t dim, const int64_t* strides, const int64_t* positions, \
                              const int64_t* position_strides, const profk_rotary_t* how, void* stream, void* out) {                                   \
        return rotary<ELEM>((const ELEM*)x, outer, inner, heads, dim, strides, positions, position_strides, how, stream, (ELEM*)out);                  \
    }                                                                                                                                                  \
    int profk_pages_append_rotary_##SUFFIX(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides, const void* v,            \
                                           const int64_t* v_strides, void* k_pages, void* v_pages, const profk_page_strides_t* kp,                     \
                                           const profk_page_strides_t* vp, const int32_t* tables, int64_t table_stride, const int32_t* lengths,        \
                                           const int32_t* starts, int64_t seqs, int64_t rows, int64_t heads, int64_t kv_heads, int64_t dim,            \
                                           int64_t page_size, int64_t pages, int64_t width, const int64_t* positions, const int64_t* position_strides, \
                                           const profk_rotary_t* how, void* stream, void* out_q) {                                                     \
        return append_rotary<ELEM>((const ELEM*)q, q_strides, (const ELEM*)k, k_strides, (const ELEM*)v, v_strides, (ELEM*)k_pages, (ELEM*)v_pages,    \
                                   kp, vp, tables, table_stride, lengths, starts, seqs, rows, heads, kv_heads, dim, page_size, pages, width,           \
                                   positions, position_strides, how, stream, (ELEM*)out_q);                                                            \
    }                                                                                                                                                  \
    int profk_adjust_logits_##SUFFIX(const void* logits, int64_t rows, int64_t V, int64_t row_stride, const profk_adjust_t* how, void* stream,         \
                                     void* out, int64_t out_row_stride) {                                                                              \
        return adjust<ELEM>((const ELEM*)logits, rows, V, row_stride, how, stream, (ELEM*)out, out_row_stride);                                        \
    }

PROFK_DEFINE_PROMPT(f32, float)
PROFK_DEFINE_PROMPT(bf16, __nv_bfloat16)
PROFK_DEFINE_PROMPT(f16, __half)

}  // extern "C"
