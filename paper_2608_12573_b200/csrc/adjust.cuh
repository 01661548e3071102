// What a sampler lays over the logits of a row before it selects.  For token v with logit x, c = its count in the answer so far:
//   y = x > 0 ? x / rho : x rho   if v was seen (prompt or answer), else x
//   y = y - (alpha_f c + alpha_p [c > 0]) + sum of v's biases;   -inf where the mask's bit is 0.
//
// Bound by HBM (each logit read and written once; in place, only the vectors that change).  What takes thought is the
// counting: histories name tokens in any order, many times.  A row belongs to a cluster of CTAs; each holds the counters of
// its slice of the vocabulary in shared memory, reads its share of the history once and adds to the counter of the CTA that
// owns the token, through distributed shared memory: integer sums, the same in any order.  A counter's top bits say "in the
// prompt" and "has a bias"; the few tokens with a bias then sum the row's list in its order, so that a token named twice gets
// the same bits every time.
#pragma once

#include "logits.cuh"

namespace profk {

constexpr int AD_THREADS = 256;
constexpr int AD_CLUSTER = 8;
constexpr int AD_MAX_BIASES = 8192;
constexpr int AD_MAX_SLICE = 32768;       // counters of a CTA; a longer vocabulary is taken in rounds
constexpr int AD_UNROLL = 4;              // vectors of a thread in flight
constexpr uint32_t AD_PROMPT = 0x80000000u, AD_BIAS = 0x40000000u, AD_COUNT = 0x3FFFFFFFu;

template <typename T>
struct AdParams {
    const T* logits;
    T* out;
    int64_t rows, row_stride, out_stride;
    uint32_t V, slice, slices;            // slice: a multiple of the vector's elements; slices: CTAs of a row without counters
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
};

struct AdBias { uint32_t token; float value; };

__device__ __forceinline__ uint32_t ad_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t ad_peer(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void ad_add(uint32_t addr, uint32_t v) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void ad_or(uint32_t addr, uint32_t v) {
    asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void ad_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}

// The entries of the row's bias list whose token exists and lies in the `slice` slots from token `lo` on (which may be
// negative), in the list's order; returns how many.
__device__ __forceinline__ int32_t ad_collect(const int64_t* tokens, const float* values, int32_t n, int64_t lo, int64_t slice, int64_t V, AdBias* list, int32_t* sums) {
    const int32_t warp = (int32_t)threadIdx.x / 32, lane = (int32_t)lane_id();
    int32_t total = 0;
    for (int32_t i0 = 0; i0 < n; i0 += AD_THREADS) {
        const int32_t i = i0 + (int32_t)threadIdx.x;
        const int64_t token = i < n ? tokens[i] : -1;
        const bool mine = token >= 0 && token < V && token >= lo && token - lo < slice;
        const uint32_t who = __ballot_sync(FULL_MASK, mine);
        if (lane == 0) sums[warp] = __popc(who);
        __syncthreads();
        int32_t before = total;
        for (int32_t w = 0; w < AD_THREADS / 32; ++w) {
            if (w < warp) before += sums[w];
            total += sums[w];
        }
        if (mine) list[before + __popc(who & ((1u << lane) - 1u))] = AdBias{(uint32_t)(token - lo), values[i]};
        __syncthreads();
    }
    return total;
}

// COUNT: there is a history or a list of biases.  Otherwise there are no clusters, and no more than one round.
template <typename T, bool COUNT>
__global__ void __launch_bounds__(AD_THREADS) adjust_logits_kernel(const AdParams<T> p) {
    constexpr int VEC = Logit<T>::VEC;
    extern __shared__ __align__(16) uint32_t counters[];                 // slice, then the biases' list
    __shared__ int32_t sums[AD_THREADS / 32];
    AdBias* list = reinterpret_cast<AdBias*>(counters + p.slice);
    const uint32_t rank = blockIdx.x % (COUNT ? (uint32_t)AD_CLUSTER : p.slices);
    const uint32_t parts = COUNT ? (uint32_t)AD_CLUSTER : p.slices;
    const int64_t row = blockIdx.x / parts;
    const T* x = p.logits + row * p.row_stride;
    T* y = p.out + row * p.out_stride;
    // vectors lie on the output's 16-byte boundaries: slot u of the row is token u - shift
    const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(y) % 16 / sizeof(T));
    const bool alike = reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T) == shift, in_place = (const T*)y == x;
    const int64_t slots = (int64_t)p.V + shift;
    const uint32_t* mask = p.mask ? p.mask + row * p.mask_stride : nullptr;
    bool waited = false;
    for (int64_t round = 0; round < slots; round += (int64_t)p.slice * parts) {
        const int64_t u0 = round + (int64_t)rank * p.slice;              // this CTA's slots: [u0, u0 + slice)
        int32_t listed = 0;
        float rho = 1.0f, alpha_f = 0.0f, alpha_p = 0.0f;
        if constexpr (COUNT) {
            __syncthreads();
            for (uint32_t i = threadIdx.x * 4; i < p.slice; i += AD_THREADS * 4) *reinterpret_cast<uint4*>(counters + i) = make_uint4(0, 0, 0, 0);
            if (!waited) { pdl_wait(); pdl_launch_dependents(); waited = true; }
            ad_cluster_sync();
            if (p.tokens) {
                const int64_t* tokens = p.tokens + row * p.token_stride;
                int64_t n = p.lengths ? (int64_t)p.lengths[row] : p.history;
                n = max((int64_t)0, min(n, p.history));
                const int64_t prompt = p.prompts ? (int64_t)p.prompts[row] : 0;
                const uint32_t here = ad_smem(counters);
                for (int64_t i0 = (int64_t)rank * AD_THREADS; i0 < n; i0 += (int64_t)AD_CLUSTER * AD_THREADS * AD_UNROLL) {
                    int64_t token[AD_UNROLL];
#pragma unroll
                    for (int j = 0; j < AD_UNROLL; ++j) {
                        const int64_t i = i0 + (int64_t)j * AD_CLUSTER * AD_THREADS + threadIdx.x;
                        token[j] = i < n ? tokens[i] : -1;
                    }
#pragma unroll
                    for (int j = 0; j < AD_UNROLL; ++j) {
                        if (token[j] < 0 || token[j] >= (int64_t)p.V) continue;
                        const int64_t u = token[j] + shift - round;
                        if (u < 0 || u >= (int64_t)p.slice * AD_CLUSTER) continue;
                        const uint32_t owner = (uint32_t)u / p.slice, at = ad_peer(here + ((uint32_t)u - owner * p.slice) * 4u, owner);
                        if (i0 + (int64_t)j * AD_CLUSTER * AD_THREADS + threadIdx.x < prompt) ad_or(at, AD_PROMPT);
                        else ad_add(at, 1u);
                    }
                }
            }
            ad_cluster_sync();
            rho = p.repetition ? p.repetition[row] : p.repetition_value;
            alpha_f = p.frequency ? p.frequency[row] : p.frequency_value;
            alpha_p = p.presence ? p.presence[row] : p.presence_value;
            if (p.bias_tokens) {
                listed = ad_collect(p.bias_tokens + row * p.bias_token_stride, p.bias_values + row * p.bias_value_stride, p.biases, u0 - shift,
                                    p.slice, p.V, list, sums);
                for (int32_t i = (int32_t)threadIdx.x; i < listed; i += AD_THREADS) atomicOr(&counters[list[i].token], AD_BIAS);
                __syncthreads();
            }
        } else {
            pdl_wait();
            pdl_launch_dependents();
        }
        auto adjusted = [&](float v, uint32_t c, uint32_t at) {
            if (c == 0u) return v;
            const float count = (float)(c & AD_COUNT);
            if (c & ~AD_BIAS) v = v > 0.0f ? v / rho : v * rho;
            if (count > 0.0f) v -= alpha_f * count + alpha_p;
            if (c & AD_BIAS) {
                float sum = 0.0f;
                for (int32_t i = 0; i < listed; ++i)
                    if (list[i].token == at) sum += list[i].value;
                v += sum;
            }
            return v;
        };
        const int64_t end = min((int64_t)p.slice, slots - u0);           // slots of this CTA that exist
        for (int64_t s0 = (int64_t)threadIdx.x * VEC; s0 < end; s0 += (int64_t)AD_THREADS * VEC * AD_UNROLL) {
            uint4 raw[AD_UNROLL];
            uint32_t allowed[AD_UNROLL];
            bool whole[AD_UNROLL], touched[AD_UNROLL];                   // a vector of existing tokens, and of the input too; one that a counter names
#pragma unroll
            for (int j = 0; j < AD_UNROLL; ++j) {
                const int64_t s = s0 + (int64_t)j * AD_THREADS * VEC, v = u0 + s - shift;
                const bool inside = s < end && v >= 0 && v + VEC <= (int64_t)p.V;
                whole[j] = inside && alike;
                allowed[j] = (1u << VEC) - 1u;
                if (mask && inside) {
                    const uint32_t low = mask[v >> 5], bit = (uint32_t)v & 31u;
                    const uint32_t high = bit + VEC > 32u ? mask[(v >> 5) + 1] : 0u;
                    allowed[j] &= __funnelshift_r(low, high, bit);
                }
                touched[j] = false;
                if constexpr (COUNT) {
                    if (inside) {
#pragma unroll
                        for (int i = 0; i < VEC; i += 4) {
                            const uint4 c = *reinterpret_cast<const uint4*>(counters + s + i);
                            touched[j] |= (c.x | c.y | c.z | c.w) != 0u;
                        }
                    }
                }
                const bool same = !touched[j] && allowed[j] == (1u << VEC) - 1u;
                if (whole[j] && allowed[j] && !(in_place && same)) raw[j] = ld_once_u4(x + v);
            }
#pragma unroll
            for (int j = 0; j < AD_UNROLL; ++j) {
                const int64_t s = s0 + (int64_t)j * AD_THREADS * VEC, v = u0 + s - shift;
                if (s >= end) continue;
                if (whole[j]) {
                    if (!touched[j] && allowed[j] == (1u << VEC) - 1u) {
                        if (!in_place) st_stream_u4(y + v, raw[j]);
                        continue;
                    }
                    if (allowed[j] == 0u) {
                        st_stream_u4(y + v, Logit<T>::masked());
                        continue;
                    }
                    float f[VEC];
                    Logit<T>::unpack(raw[j], f);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        if constexpr (COUNT) {
                            if (touched[j]) f[i] = adjusted(f[i], counters[s + i], (uint32_t)(s + i));
                        }
                        if (!(allowed[j] >> i & 1u)) f[i] = -INFINITY;
                    }
                    st_stream_u4(y + v, Logit<T>::pack(f));
                } else {
                    for (int i = 0; i < VEC; ++i) {
                        const int64_t t = v + i;
                        if (t < 0 || t >= (int64_t)p.V) continue;
                        T e = x[t];
                        if constexpr (COUNT) {
                            if (counters[s + i]) e = Logit<T>::from_float(adjusted(Logit<T>::to_float(e), counters[s + i], (uint32_t)(s + i)));
                        }
                        if (mask && !(mask[t >> 5] >> (t & 31) & 1u)) e = Logit<T>::from_float(-INFINITY);
                        y[t] = e;
                    }
                }
            }
        }
    }
}

}  // namespace profk
