// What a sampler lays over the logits of a row before it selects.  For token v with logit x, c = its count in the answer so far:
//   y = x > 0 ? x / rho : x rho   if v was seen (prompt or answer), else x
//   y = y - (alpha_f c + alpha_p [c > 0]) + sum of v's biases;   -inf where the mask's bit is 0.
//
// Bound by HBM (each logit read and written once; in place, only what changes).  One kernel streams the rows through with the
// mask; a second goes back to the few tokens that a history or a list of biases names (it counts while the first one ends).
// (One kernel that looked at every element's counter while streaming: in a warp some lane always has a named one, and the
// division is then done for all; 256 rows of 131071 bf16 with 4096 tokens of history each 95 us.  One kernel that streamed a
// slice and then went back: 68, the SMs idle while they count and list.  Now 64 with 30 biases and a mask, of which the stream takes 25.)
//
// Histories name tokens in any order, many times.  A CTA of the second kernel has a slice of a row's vocabulary: it goes over
// the row's whole history (which comes from L2 but for the first time) and counts its own tokens in shared memory: integer
// sums, the same in any order.  (CTAs of a cluster that each read a share and counted for one another were slower: a remote
// count takes 14 cycles of an SM; 116 us.)  Then the counters that are not zero are gathered into a list, so that every lane
// has a token to adjust and many reads are in flight.  A token with biases is adjusted by the entry that names it first, in
// the list's order, and so gets the same bits every time.
#pragma once

#include "logits.cuh"

namespace profk {

constexpr int AD_THREADS = 256, AD_UNROLL = 4;         // of the stream; vectors of a thread in flight
constexpr int AD_NAMED_THREADS = 512, AD_PAIRS = 4, AD_HISTORY = 8;        // of the second kernel; pairs of tokens of the history, and named tokens, of a thread in flight
constexpr int AD_MAX_BIASES = 8192;
constexpr uint32_t AD_PROMPT = 0x80000000u, AD_COUNT = 0x7FFFFFFFu;           // a counter: whether the prompt names the token, its count in the answer
constexpr int64_t AD_NARROW = 32768;      // tokens of a history from which counters of 16 bits may not do

// Counters of a slice, 16 or 32 bits each: the highest bit is for the prompt.
template <int BITS>
struct AdCounters {
    uint32_t* words;
    static constexpr int PER = BITS == 16 ? 2 : 1;                       // counters of a word
    static constexpr uint32_t SLICE = BITS == 16 ? 32768 : 16384;        // tokens of a CTA at most
    static __host__ __device__ constexpr size_t bytes(size_t slice) { return slice * (BITS / 8); }
    __device__ __forceinline__ void add(uint32_t token) const {
        if constexpr (BITS == 16) atomicAdd(words + token / 2, 1u << (token % 2 * 16));
        else atomicAdd(words + token, 1u);
    }
    __device__ __forceinline__ void prompt(uint32_t token) const {
        if constexpr (BITS == 16) atomicOr(words + token / 2, 0x8000u << (token % 2 * 16));
        else atomicOr(words + token, AD_PROMPT);
    }
    __device__ __forceinline__ uint32_t of(uint32_t token) const {
        if constexpr (BITS == 16) {
            const uint32_t c = words[token / 2] >> (token % 2 * 16) & 0xFFFFu;
            return (c & 0x8000u) << 16 | (c & 0x7FFFu);
        } else {
            return words[token];
        }
    }
    __device__ __forceinline__ void clear(uint32_t token) const {
        if constexpr (BITS == 16) atomicAnd(words + token / 2, 0xFFFF0000u >> (token % 2 * 16));
        else words[token] = 0u;
    }
};

template <typename T>
struct AdParams {
    const T* logits;
    T* out;
    int64_t rows, row_stride, out_stride;
    uint32_t V, slice, slices;            // tokens of a CTA, CTAs of a row; of each kernel its own
    const int64_t* tokens;                // null: no history
    int64_t history, token_stride;
    const int32_t* lengths;               // null: all of it
    const int32_t* prompts;               // null: 0
    const float* repetition;              // per row; null: the number below
    const float* frequency;
    const float* presence;
    float repetition_value, frequency_value, presence_value;
    const int64_t* bias_tokens;           // null: none
    const float* bias_values;
    int32_t biases;
    int64_t bias_token_stride, bias_value_stride;
    const uint32_t* mask;                 // null: all allowed
    int64_t mask_stride;
    bool behind_stream;                   // of the second kernel: the first runs before it
};

struct AdBias { uint32_t token; float value; };

// The entries of the row's bias list whose token exists and lies in the `slice` slots from token `lo` on (which may be
// negative), in the list's order; returns how many.
__device__ __forceinline__ int32_t ad_collect(const int64_t* tokens, const float* values, int32_t n, int64_t lo, int64_t slice, int64_t V, AdBias* list, int32_t* sums) {
    const int32_t warp = (int32_t)threadIdx.x / 32, lane = (int32_t)lane_id();
    int32_t total = 0;
    for (int32_t i0 = 0; i0 < n; i0 += AD_NAMED_THREADS) {
        const int32_t i = i0 + (int32_t)threadIdx.x;
        const int64_t token = i < n ? tokens[i] : -1;
        const bool mine = token >= 0 && token < V && token >= lo && token - lo < slice;
        const uint32_t who = __ballot_sync(FULL_MASK, mine);
        if (lane == 0) sums[warp] = __popc(who);
        __syncthreads();
        int32_t before = total;
        for (int32_t w = 0; w < AD_NAMED_THREADS / 32; ++w) {
            if (w < warp) before += sums[w];
            total += sums[w];
        }
        if (mine) list[before + __popc(who & ((1u << lane) - 1u))] = AdBias{(uint32_t)(token - lo), values[i]};
        __syncthreads();
    }
    return total;
}

// A vector with -inf in the places that are not allowed; the others keep their bits.
template <typename T>
__device__ __forceinline__ uint4 ad_masked(const uint4& v, uint32_t allowed) {
    const uint4 off = Logit<T>::masked();
    uint4 r;
    auto word = [&](uint32_t x, uint32_t none, int i) {
        if constexpr (sizeof(T) == 4) return allowed >> i & 1u ? x : none;
        const uint32_t keep = (allowed >> (2 * i) & 1u ? 0x0000FFFFu : 0u) | (allowed >> (2 * i + 1) & 1u ? 0xFFFF0000u : 0u);
        return (x & keep) | (none & ~keep);
    };
    r.x = word(v.x, off.x, 0);
    r.y = word(v.y, off.y, 1);
    r.z = word(v.z, off.z, 2);
    r.w = word(v.w, off.w, 3);
    return r;
}

template <typename T>
__global__ void __launch_bounds__(AD_THREADS) adjust_stream_kernel(const AdParams<T> p) {
    constexpr int VEC = Logit<T>::VEC;
    constexpr uint32_t ALL = (1u << VEC) - 1u;
    const int64_t row = blockIdx.x / p.slices;
    const T* x = p.logits + row * p.row_stride;
    T* y = p.out + row * p.out_stride;
    // vectors lie on the output's 16-byte boundaries: slot u of the row is token u - shift
    const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(y) % 16 / sizeof(T));
    const bool alike = reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T) == shift, in_place = (const T*)y == x;
    const int64_t u0 = (int64_t)(blockIdx.x - (uint32_t)row * p.slices) * p.slice, slots = (int64_t)p.V + shift;
    const uint32_t* mask = p.mask ? p.mask + row * p.mask_stride : nullptr;
    pdl_wait();
    pdl_launch_dependents();
    const int64_t end = min((int64_t)p.slice, slots - u0);               // slots of this CTA that exist
    for (int64_t s0 = (int64_t)threadIdx.x * VEC; s0 < end; s0 += (int64_t)AD_THREADS * VEC * AD_UNROLL) {
        uint4 raw[AD_UNROLL];
        uint32_t allowed[AD_UNROLL];
        bool whole[AD_UNROLL];                                           // a vector of existing tokens, and of the input too
#pragma unroll
        for (int j = 0; j < AD_UNROLL; ++j) {
            const int64_t s = s0 + (int64_t)j * AD_THREADS * VEC, v = u0 + s - shift;
            whole[j] = alike && s < end && v >= 0 && v + VEC <= (int64_t)p.V;
            allowed[j] = ALL;
            if (mask && whole[j]) {
                const uint32_t low = mask[v >> 5], bit = (uint32_t)v & 31u;
                const uint32_t high = bit + VEC > 32u ? mask[(v >> 5) + 1] : 0u;
                allowed[j] &= __funnelshift_r(low, high, bit);
            }
            if (whole[j] && allowed[j] && !(in_place && allowed[j] == ALL)) raw[j] = ld_once_u4(x + v);
        }
#pragma unroll
        for (int j = 0; j < AD_UNROLL; ++j) {
            const int64_t s = s0 + (int64_t)j * AD_THREADS * VEC, v = u0 + s - shift;
            if (s >= end) continue;
            if (!whole[j]) {
                for (int64_t t = max(v, (int64_t)0); t < min(v + VEC, (int64_t)p.V); ++t) {
                    if (mask && !(mask[t >> 5] >> (t & 31) & 1u)) y[t] = Logit<T>::from_float(-INFINITY);
                    else if (!in_place) y[t] = x[t];
                }
            } else if (allowed[j] == ALL) {
                if (!in_place) st_stream_u4(y + v, raw[j]);
            } else {
                st_stream_u4(y + v, allowed[j] == 0u ? Logit<T>::masked() : ad_masked<T>(raw[j], allowed[j]));
            }
        }
    }
}

template <typename T, int BITS>
__global__ void __launch_bounds__(AD_NAMED_THREADS, BITS == 16 ? 3 : 2) adjust_named_kernel(const AdParams<T> p) {
    extern __shared__ __align__(16) uint32_t memory[];                   // counters, the biases' list, the named tokens' list
    __shared__ int32_t sums[AD_NAMED_THREADS / 32];
    const AdCounters<BITS> counters{memory};
    const int64_t row = blockIdx.x / p.slices;
    const T* x = p.logits + row * p.row_stride;
    T* y = p.out + row * p.out_stride;
    const uint32_t* mask = p.mask ? p.mask + row * p.mask_stride : nullptr;
    // its tokens: `held` of them from `from` on
    const int64_t from = (int64_t)(blockIdx.x - (uint32_t)row * p.slices) * p.slice;
    const uint32_t held = (uint32_t)min((int64_t)p.slice, (int64_t)p.V - from);
    // what is read until the wait is inputs that the kernel before this one (the stream) had waited for, and does not write
    if (p.tokens) {
        for (uint32_t i = threadIdx.x * 16; i < AdCounters<BITS>::bytes(p.slice); i += AD_NAMED_THREADS * 16) *reinterpret_cast<uint4*>(memory + i / 4) = make_uint4(0, 0, 0, 0);
        if (!p.behind_stream) pdl_wait();
        const int64_t* tokens = p.tokens + row * p.token_stride;
        const int64_t n = max((int64_t)0, min(p.lengths ? (int64_t)p.lengths[row] : p.history, p.history));
        const int64_t prompt = p.prompts ? (int64_t)p.prompts[row] : 0;
        __syncthreads();
        // f(token - from) for the tokens [begin, end) of the history that are this CTA's: two to a 16-byte load, in 32 bits from there
        const uint32_t base = (uint32_t)from;
        auto scan = [&](int64_t begin, int64_t end, auto&& f) {
            if (begin >= end) return;
            auto one = [&](uint32_t low, uint32_t high) {
                if (high == 0u && low - base < held) f(low - base);
            };
            const int64_t* at = tokens + begin;
            const int64_t head = reinterpret_cast<uintptr_t>(at) % 16 != 0 ? 1 : 0, pairs = (end - begin - head) / 2, rest = end - begin - head - 2 * pairs;
            auto single = [&](const int64_t* t) { one((uint32_t)*t, (uint32_t)((uint64_t)*t >> 32)); };
            if (threadIdx.x == 0 && head) single(at);
            if (threadIdx.x == 32 && rest) single(tokens + end - 1);
            const uint4* two = reinterpret_cast<const uint4*>(at + head);
            for (int64_t i0 = (int64_t)threadIdx.x; i0 < pairs; i0 += (int64_t)AD_NAMED_THREADS * AD_PAIRS) {
                uint4 v[AD_PAIRS];
#pragma unroll
                for (int j = 0; j < AD_PAIRS; ++j) {
                    const int64_t i = i0 + (int64_t)j * AD_NAMED_THREADS;
                    v[j] = i < pairs ? __ldg(two + i) : make_uint4(0u, ~0u, 0u, ~0u);
                }
#pragma unroll
                for (int j = 0; j < AD_PAIRS; ++j) {
                    one(v[j].x, v[j].y);
                    one(v[j].z, v[j].w);
                }
            }
        };
        const int64_t split = max((int64_t)0, min(prompt, n));
        scan(0, split, [&](uint32_t token) { counters.prompt(token); });
        scan(split, n, [&](uint32_t token) { counters.add(token); });
        __syncthreads();
    } else if (!p.behind_stream) {
        pdl_wait();
    }
    const float rho = p.repetition ? p.repetition[row] : p.repetition_value;
    const float alpha_f = p.frequency ? p.frequency[row] : p.frequency_value, alpha_p = p.presence ? p.presence[row] : p.presence_value;
    auto penalised = [&](float v, uint32_t c) {
        if (c) v = v > 0.0f ? v / rho : v * rho;
        if (c & AD_COUNT) v -= alpha_f * (float)(c & AD_COUNT) + alpha_p;
        return v;
    };
    auto is_allowed = [&](int64_t t) { return !mask || (mask[t >> 5] >> (t & 31) & 1u); };
    AdBias* list = reinterpret_cast<AdBias*>(memory + (p.tokens ? AdCounters<BITS>::bytes(p.slice) / 4 : 0));
    int32_t listed = 0;
    if (p.bias_tokens) listed = ad_collect(p.bias_tokens + row * p.bias_token_stride, p.bias_values + row * p.bias_value_stride, p.biases, from, held, p.V, list, sums);
    if (p.behind_stream) pdl_wait();                                     // (what the stream writes comes first)
    pdl_launch_dependents();
    for (int32_t i = (int32_t)threadIdx.x; i < listed; i += AD_NAMED_THREADS) {
        const uint32_t token = list[i].token;
        bool first = true;
        for (int32_t j = 0; first && j < i; ++j) first = list[j].token != token;
        if (!first) continue;
        const int64_t t = from + token;
        if (is_allowed(t)) {
            float v = penalised(Logit<T>::to_float(x[t]), p.tokens ? counters.of(token) : 0u), sum = 0.0f;
            for (int32_t j = i; j < listed; ++j)
                if (list[j].token == token) sum += list[j].value;
            y[t] = Logit<T>::from_float(v + sum);
        }
        if (p.tokens) counters.clear(token);                             // its penalties are in
    }
    if (!p.tokens) return;
    uint16_t* named = reinterpret_cast<uint16_t*>(list + p.biases);
    constexpr int PER = 4 * AdCounters<BITS>::PER;                       // counters of 16 bytes
    __syncthreads();
    if (threadIdx.x == 0) sums[0] = 0;
    __syncthreads();
    for (uint32_t i0 = 0; i0 < p.slice; i0 += AD_NAMED_THREADS * PER) {
        const uint32_t i = i0 + threadIdx.x * PER;
        const uint4 c = i < p.slice ? *reinterpret_cast<const uint4*>(memory + i / AdCounters<BITS>::PER) : make_uint4(0, 0, 0, 0);
        const uint32_t word[4] = {c.x, c.y, c.z, c.w};
        uint32_t which = 0;                                              // bits: this thread's counters that are not zero
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (BITS == 16) which |= ((word[k] & 0xFFFFu) != 0u ? 1u << 2 * k : 0u) | ((word[k] >> 16) != 0u ? 2u << 2 * k : 0u);
            else which |= word[k] != 0u ? 1u << k : 0u;
        }
        if (!which) continue;
        int32_t at = atomicAdd(&sums[0], __popc(which));                 // (in any order: a token's result does not depend on its place)
        for (; which; which &= which - 1u) named[at++] = (uint16_t)(i + (uint32_t)__ffs((int)which) - 1u);
    }
    __syncthreads();
    const int32_t found = sums[0];
    for (int32_t i0 = (int32_t)threadIdx.x; i0 < found; i0 += AD_NAMED_THREADS * AD_HISTORY) {
        uint32_t token[AD_HISTORY];
        T e[AD_HISTORY];
        bool on[AD_HISTORY];
#pragma unroll
        for (int j = 0; j < AD_HISTORY; ++j) {
            on[j] = i0 + j * AD_NAMED_THREADS < found;
            token[j] = on[j] ? named[i0 + j * AD_NAMED_THREADS] : 0u;
            on[j] = on[j] && is_allowed(from + token[j]);
            if (on[j]) e[j] = x[from + token[j]];
        }
#pragma unroll
        for (int j = 0; j < AD_HISTORY; ++j)
            if (on[j]) y[from + token[j]] = Logit<T>::from_float(penalised(Logit<T>::to_float(e[j]), counters.of(token[j])));
    }
}

}  // namespace profk
