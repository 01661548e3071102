// Log probabilities of given tokens, entropy and top alternatives of every row of a logits matrix, in one read of it,
// and their gradient.
//
// With z = x / T, m = max z and s = sum e^(z - m) over a row:   lse = m + ln s,   ln p_v = z_v - lse,
//   H = -sum p ln p = ln s - (1/s) sum e^(z - m) (z - m).
// A part of a row is described by (m, s, t), t = sum e^(z - m) (x - mx) with mx its largest logit; two parts join by
// moving both to the larger maximum, so every thread keeps a triple of its own and they are joined in a fixed order at
// the end of the row.  T only enters as a factor of the exponent: e^(z - m) = 2^((x - mx) log2(e) / T).
//
// The k largest logits are found on the way: a float bound is compared with the largest element of each batch, elements
// at or above it are appended to a list in shared memory, and when the list fills the k best of it raise the bound.
#pragma once

#include <cooperative_groups.h>

#include "logits.cuh"

namespace profk {

namespace cg = cooperative_groups;

constexpr int LP_THREADS = 512;
constexpr int LP_UNROLL = 4;              // 16-byte vectors per thread and batch
constexpr int LP_STAGES = 3;              // batches in flight or in hand per thread
constexpr uint32_t LP_CAP = 1024;         // records the candidate list holds
constexpr uint32_t LP_HIGH = 512;        // beyond this many the list is cut back to its k best
constexpr uint32_t LP_MAX_K = 128;        // most alternatives
constexpr uint32_t LP_SLACK = 32;         // a selection may stop with up to k + LP_SLACK records in hand

struct LpParams {
    const void* logits;
    int64_t rows, row_stride;
    uint32_t V, k;
    float scale;                          // 1 / T
    const int64_t* tokens;                // may be null
    float* logprob;
    float* lse;
    float* lse_rest;                      // may be null
    float* entropy;
    float* top_logprobs;
    int64_t* top_tokens;
};

struct LpStats { float m, s, t; };

// Both parts moved to the larger maximum; c = log2(e) / T.
__device__ __forceinline__ LpStats lp_join(const LpStats& a, const LpStats& b, float c) {
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf(a.m - m, FAR_BELOW), db = fmaxf(b.m - m, FAR_BELOW);
    const float fa = exp2_approx(da * c), fb = exp2_approx(db * c);
    return LpStats{m, fa * a.s + fb * b.s, fa * fmaf(da, a.s, a.t) + fb * fmaf(db, b.s, b.t)};
}

struct LpShared {
    uint64_t cand[LP_CAP];
    uint64_t best[LP_MAX_K + LP_SLACK];
    uint32_t part[2][LP_THREADS / 32];
    uint32_t lo[LP_THREADS / 32], hi[LP_THREADS / 32];
    LpStats stats[LP_THREADS / 32];
    uint32_t count, fill;
    uint64_t limit;                       // records above it are no longer of interest
    float bound;                          // elements below it are no longer of interest
    float row_max, row_log;               // of the finished row: largest logit, ln s
};

// Sum over the CTA of one number per thread; `turn` alternates between calls, so that one barrier is enough.
__device__ __forceinline__ uint32_t lp_block_sum(uint32_t v, LpShared& sh, int turn) {
    const uint32_t w = __reduce_add_sync(FULL_MASK, v);
    if (lane_id() == 0) sh.part[turn][threadIdx.x >> 5] = w;
    __syncthreads();
    const unsigned lane = lane_id();
    return __reduce_add_sync(FULL_MASK, lane < LP_THREADS / 32 ? sh.part[turn][lane] : 0u);
}

// The least limit found (by halving the interval of the records' value words, then of their index words) such that at
// least k and at most `most` of the n records in `a` are <= it; fewer than k valid records (~0 is none): all of them.
// All threads call it and get the same answer; a barrier must lie between the last write to `a` and the call.
__device__ __forceinline__ uint64_t lp_find_limit(const uint64_t* a, uint32_t n, uint32_t k, uint32_t most, LpShared& sh) {
    const unsigned tid = threadIdx.x, lane = lane_id();
    uint32_t lo = 0xFFFFFFFFu, hi = 0u, valid = 0;
    for (uint32_t i = tid; i < n; i += LP_THREADS) {
        const uint64_t r = a[i];
        if (r != ~0ull) {
            const uint32_t h = (uint32_t)(r >> 32);
            lo = min(lo, h);
            hi = max(hi, h);
            ++valid;
        }
    }
    lo = __reduce_min_sync(FULL_MASK, lo);
    hi = __reduce_max_sync(FULL_MASK, hi);
    if (lane == 0) { sh.lo[tid >> 5] = lo; sh.hi[tid >> 5] = hi; }
    const uint32_t total = lp_block_sum(valid, sh, 0);      // its barrier also covers lo and hi
    if (total <= most) return ~0ull - 1;
    lo = __reduce_min_sync(FULL_MASK, lane < LP_THREADS / 32 ? sh.lo[lane] : 0xFFFFFFFFu);
    hi = __reduce_max_sync(FULL_MASK, lane < LP_THREADS / 32 ? sh.hi[lane] : 0u);
    int turn = 1;
    // smallest value word `lo` with at least k records at or below it
    while (lo < hi) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        uint32_t c = 0;
        for (uint32_t i = tid; i < n; i += LP_THREADS) c += (uint32_t)(a[i] >> 32) <= mid && a[i] != ~0ull;
        c = lp_block_sum(c, sh, turn);
        turn ^= 1;
        if (c >= k) {
            hi = mid;
            if (c <= most) return ((uint64_t)mid << 32) | 0xFFFFFFFFull;
        } else {
            lo = mid + 1;
        }
    }
    const uint32_t word = lo;
    uint32_t ilo = 0, ihi = 0xFFFFFFFFu;
    while (ilo < ihi) {
        const uint32_t mid = ilo + ((ihi - ilo) >> 1);
        const uint64_t limit = ((uint64_t)word << 32) | mid;
        uint32_t c = 0;
        for (uint32_t i = tid; i < n; i += LP_THREADS) c += a[i] <= limit;
        c = lp_block_sum(c, sh, turn);
        turn ^= 1;
        if (c >= k) {
            ihi = mid;
            if (c <= most) break;
        } else {
            ilo = mid + 1;
        }
    }
    __syncthreads();
    return ((uint64_t)word << 32) | ihi;
}

// Copies the records <= limit of a[0, n) into sh.best (at most `room` of them) and returns how many there are.
__device__ __forceinline__ uint32_t lp_collect(const uint64_t* a, uint32_t n, uint64_t limit, uint32_t room, LpShared& sh) {
    __syncthreads();
    if (threadIdx.x == 0) sh.fill = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += LP_THREADS) {
        const uint64_t r = a[i];
        if (r <= limit) {
            const uint32_t pos = atomicAdd(&sh.fill, 1u);
            if (pos < room) sh.best[pos] = r;
        }
    }
    __syncthreads();
    return min(sh.fill, room);
}

// Cuts the candidate list back to its k best and raises the bound above the worst of them: what follows has higher
// indices, so that an equal element no longer counts.
__device__ __forceinline__ void lp_cut_list(uint32_t stored, uint32_t k, LpShared& sh) {
    // exactly k: the k-th record is then the bound for everything that follows
    const uint64_t limit = lp_find_limit(sh.cand, stored, k, k, sh);
    const uint32_t m = lp_collect(sh.cand, stored, limit, LP_MAX_K + LP_SLACK, sh);
    for (uint32_t i = threadIdx.x; i < m; i += LP_THREADS) sh.cand[i] = sh.best[i];
    if (threadIdx.x == 0) {
        sh.count = m;
        sh.limit = limit;
        sh.bound = __uint_as_float(bits32_from_key(~(uint32_t)(limit >> 32) + 1u));
    }
    __syncthreads();
}

template <typename T>
__device__ __forceinline__ uint64_t lp_record(float x, uint32_t idx) { return make_record(key_from_bits32(float_bits_exact(x)), idx); }

template <typename T>
__device__ __forceinline__ void lp_append(float x, uint32_t idx, LpShared& sh) {
    const uint64_t rec = lp_record<T>(x, idx);
    if (rec <= sh.limit) {
        const uint32_t pos = atomicAdd(&sh.count, 1u);
        if (pos < LP_CAP) sh.cand[pos] = rec;
    }
}

__device__ __forceinline__ void lp_cp_async16(uint32_t smem, const void* gmem) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
}
__device__ __forceinline__ void lp_cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void lp_cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where the vectors of one row's share lie.
template <typename T>
struct LpShare {
    const T* x;            // row start
    uint32_t head;         // elements before the first 16-byte boundary
    uint32_t nvec;         // vectors of the row
    uint32_t v0, v1;       // this CTA's vectors
    __device__ __forceinline__ void set(const LpParams& p, int64_t row, uint32_t part, uint32_t parts) {
        x = reinterpret_cast<const T*>(p.logits) + row * p.row_stride;
        const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(x) & 15u);
        head = min(p.V, mis ? (16u - mis) / (uint32_t)sizeof(T) : 0u);
        nvec = (p.V - head) / Logit<T>::VEC;
        v0 = (uint32_t)((uint64_t)nvec * part / parts);
        v1 = (uint32_t)((uint64_t)nvec * (part + 1) / parts);
    }
    __device__ __forceinline__ const T* vec(uint32_t v) const { return x + head + (size_t)v * Logit<T>::VEC; }
};

// One cluster of `parts` CTAs takes a row at a time (parts = 1: a plain CTA).  The vectors of the row come through a ring
// in shared memory that each thread fills and empties for itself (cp.async, no barrier), and that runs on into the next
// row, so that HBM stays busy while a row is finished.
template <typename T, bool ENT, bool TOPK>
__global__ void __launch_bounds__(LP_THREADS, 2) logprobs_kernel(const LpParams p) {
    constexpr int VEC = Logit<T>::VEC, U = LP_UNROLL;
    constexpr uint32_t STEP = LP_THREADS * U;
    extern __shared__ __align__(16) unsigned char lp_dyn[];
    __shared__ LpShared sh;
    uint4* ring = reinterpret_cast<uint4*>(lp_dyn);                               // [LP_STAGES][U][LP_THREADS]
    const uint32_t lim = TOPK ? p.k + LP_SLACK : 0;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t parts = cluster.num_blocks(), part = cluster.block_rank();
    // what the parts of a row hand to the first of them: two sets, used in turn
    uint64_t* in_recs = reinterpret_cast<uint64_t*>(ring + (size_t)LP_STAGES * U * LP_THREADS);   // [2][parts][lim]
    LpStats* in_stats = reinterpret_cast<LpStats*>(in_recs + (parts > 1 ? 2 * (size_t)parts * lim : 0));   // [2][parts]

    const unsigned tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    const int64_t first = blockIdx.x / parts, stride = gridDim.x / parts;
    const float c = p.scale * LOG2E;
    pdl_wait();
    pdl_launch_dependents();
    if (parts > 1) cluster.sync();                                                // every CTA of the cluster has started

    // the loading side runs LP_STAGES - 1 batches ahead of the working side
    int64_t load_row = first;
    LpShare<T> ld;
    uint32_t load_v = 0;
    int load_stage = 0;
    if (load_row < p.rows) { ld.set(p, load_row, part, parts); load_v = ld.v0; }
    const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
    auto load_batch = [&]() {
        if (load_row < p.rows) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t v = load_v + u * LP_THREADS + tid;
                if (v < ld.v1) lp_cp_async16(ring_addr + ((load_stage * U + u) * LP_THREADS + tid) * 16u, ld.vec(v));
            }
            load_v += STEP;
            if (load_v >= ld.v1) {
                load_row += stride;
                if (load_row < p.rows) { ld.set(p, load_row, part, parts); load_v = ld.v0; }
            }
        }
        lp_cp_commit();
        load_stage = load_stage + 1 == LP_STAGES ? 0 : load_stage + 1;
    };
#pragma unroll
    for (int s = 0; s < LP_STAGES - 1; ++s) load_batch();

    int stage = 0;
    uint32_t turn = 0;                                                            // of the hand-over sets
    for (int64_t row = first; row < p.rows; row += stride) {
        LpShare<T> mine;
        mine.set(p, row, part, parts);
        LpStats st{LOWEST, 0.f, 0.f};
        if constexpr (TOPK) {
            if (tid == 0) { sh.count = 0; sh.limit = ~0ull - 1; sh.bound = -INFINITY; }
            __syncthreads();
        }
        auto one = [&](float x) {                                                 // a single element
            if (x > st.m) {
                const float d = fmaxf(st.m - x, FAR_BELOW), f = exp2_approx(d * c);
                st.t = f * fmaf(d, st.s, st.t);
                st.s *= f;
                st.m = x;
            }
            const float d = x - st.m, e = exp2_approx(d * c);
            st.s += e;
            if constexpr (ENT) st.t = fmaf(e, fmaxf(d, FAR_BELOW), st.t);
        };
        // elements before the first whole vector
        if (part == 0 && tid < mine.head) {
            const float x = Logit<T>::to_float(mine.x[tid]);
            one(x);
            if (TOPK && x >= -INFINITY) lp_append<T>(x, tid, sh);
        }
        bool opening = true;
        uint32_t v = mine.v0;
        do {                                                                      // (an empty share still takes its batch)
            load_batch();
            lp_cp_wait<LP_STAGES - 1>();
            uint4 vec[U];
            float vmax[U], bmax = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = v + u * LP_THREADS + tid < mine.v1;
                vec[u] = ring[(stage * U + u) * LP_THREADS + tid];
                vmax[u] = in ? Logit<T>::vec_max(vec[u]) : -INFINITY;
                bmax = fmaxf(bmax, vmax[u]);
            }
            if (bmax > st.m) {
                const float d = fmaxf(st.m - bmax, FAR_BELOW), f = exp2_approx(d * c);
                st.t = f * fmaf(d, st.s, st.t);
                st.s *= f;
                st.m = bmax;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * LP_THREADS + tid < mine.v1) {
                    float x[VEC];
                    Logit<T>::unpack(vec[u], x);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float d = x[j] - st.m, e = exp2_approx(d * c);
                        st.s += e;
                        if constexpr (ENT) st.t = fmaf(e, fmaxf(d, FAR_BELOW), st.t);
                    }
                }
            }
            if constexpr (TOPK) {
                if (opening) {
                    // The k-th largest of the threads' maxima has k elements at or above it: a first bound, found by
                    // halving the interval of the order keys until at most k + LP_SLACK maxima reach it.
                    opening = false;
                    const uint32_t key = key_from_bits32(float_bits_exact(bmax));
                    uint32_t lo = 0x007FFFFFu, hi = 0xFF800001u;                  // keys of -inf and of +inf + 1
                    // invariant: at least k maxima have a key >= lo (every thread has at least -inf)
                    while (lo + 1 < hi) {
                        const uint32_t mid = lo + ((hi - lo) >> 1);
                        const uint32_t n = (uint32_t)__syncthreads_count(key >= mid);
                        if (n >= p.k) {
                            lo = mid;
                            if (n <= p.k + LP_SLACK) break;
                        } else {
                            hi = mid;
                        }
                    }
                    if (tid == 0) sh.bound = __uint_as_float(bits32_from_key(lo));
                    __syncthreads();
                }
                const uint32_t before = sh.count;                                 // read behind a barrier of this or the last batch
                __syncthreads();
                for (;;) {
                    const float bound = sh.bound;
                    if (bmax >= bound) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            if (vmax[u] >= bound && v + u * LP_THREADS + tid < mine.v1) {
                                float x[VEC];
                                Logit<T>::unpack(vec[u], x);
                                const uint32_t at = mine.head + (v + u * LP_THREADS + tid) * VEC;
#pragma unroll
                                for (int j = 0; j < VEC; ++j)
                                    if (x[j] >= bound) lp_append<T>(x[j], at + j, sh);
                            }
                        }
                    }
                    __syncthreads();
                    const uint32_t now = sh.count;
                    if (now <= LP_CAP) {
                        if (now > LP_HIGH) {
                            __syncthreads();
                            lp_cut_list(now, p.k, sh);
                        }
                        break;
                    }
                    // More than the list holds: the k best of what it holds bound what this batch may still add.  The
                    // batch's own records are dropped again and the batch is looked at once more under that bound.
                    __syncthreads();
                    const uint64_t limit = lp_find_limit(sh.cand, LP_CAP, p.k, p.k, sh);
                    if (tid == 0) {
                        sh.limit = limit;
                        sh.bound = __uint_as_float(bits32_from_key(~(uint32_t)(limit >> 32)));
                        sh.count = before;
                    }
                    __syncthreads();
                }
            }
            stage = stage + 1 == LP_STAGES ? 0 : stage + 1;
            v += STEP;
        } while (v < mine.v1);
        // elements behind the last whole vector (the list has room: it holds LP_HIGH records at most here)
        const uint32_t tail = mine.head + mine.nvec * VEC;
        if (part == parts - 1 && tail + tid < p.V) {
            const float x = Logit<T>::to_float(mine.x[tail + tid]);
            one(x);
            if (TOPK && x >= -INFINITY) lp_append<T>(x, tail + tid, sh);
        }

        // join the threads' parts, in a fixed order
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            LpStats o;
            o.m = __shfl_xor_sync(FULL_MASK, st.m, d);
            o.s = __shfl_xor_sync(FULL_MASK, st.s, d);
            o.t = __shfl_xor_sync(FULL_MASK, st.t, d);
            st = (lane & d) ? lp_join(o, st, c) : lp_join(st, o, c);
        }
        __syncthreads();
        if (lane == 0) sh.stats[warp] = st;
        uint32_t found = 0;
        if constexpr (TOPK) {
            __syncthreads();
            const uint32_t n = sh.count;
            const uint64_t limit = lp_find_limit(sh.cand, n, p.k, lim, sh);
            found = lp_collect(sh.cand, n, limit, lim, sh);
        }
        __syncthreads();
        if (parts > 1) {
            // hand statistics and records to the cluster's first CTA
            LpStats* to_stats = cluster.map_shared_rank(in_stats, 0) + turn * parts + part;
            uint64_t* to_recs = cluster.map_shared_rank(in_recs, 0) + ((size_t)turn * parts + part) * lim;
            if constexpr (TOPK)
                for (uint32_t i = tid; i < lim; i += LP_THREADS) to_recs[i] = i < found ? sh.best[i] : ~0ull;
            if (tid == 0) {
                LpStats all = sh.stats[0];
                for (int w = 1; w < LP_THREADS / 32; ++w) all = lp_join(all, sh.stats[w], c);
                *to_stats = all;
            }
            cluster.sync();
        }
        if (part == 0) {
            if (tid == 0) {
                LpStats all;
                if (parts > 1) {
                    all = in_stats[turn * parts];
                    for (uint32_t i = 1; i < parts; ++i) all = lp_join(all, in_stats[turn * parts + i], c);
                } else {
                    all = sh.stats[0];
                    for (int w = 1; w < LP_THREADS / 32; ++w) all = lp_join(all, sh.stats[w], c);
                }
                const bool empty = all.s == 0.f;                                  // nothing but -inf
                const float log_s = logf(all.s);
                sh.row_max = all.m;
                sh.row_log = log_s;
                // lse in two floats: one alone loses ln s beside a large maximum (all of it in a row masked with fp32's
                // lowest value), and with it the probabilities that the gradient takes from it
                const float near = empty ? -INFINITY : fmaf(all.m, p.scale, log_s);
                p.lse[row] = near;
                if (p.lse_rest) p.lse_rest[row] = isinf(near) ? 0.f : fmaf(all.m, p.scale, -near) + log_s;
                if constexpr (ENT) p.entropy[row] = empty ? 0.f : log_s - p.scale * (all.t / all.s);
                if (p.logprob) {
                    const int64_t token = p.tokens[row];
                    float lp = 0.f;                                               // no token given
                    if (token >= (int64_t)p.V) lp = NAN;
                    else if (token >= 0)
                        lp = empty ? -INFINITY
                                   : (Logit<T>::to_float((reinterpret_cast<const T*>(p.logits) + row * p.row_stride)[token]) - all.m) * p.scale - log_s;
                    p.logprob[row] = lp;
                }
            }
            if constexpr (TOPK) {
                if (parts > 1) {
                    const uint64_t* recs = in_recs + (size_t)turn * parts * lim;
                    const uint64_t limit = lp_find_limit(recs, parts * lim, p.k, lim, sh);
                    found = lp_collect(recs, parts * lim, limit, lim, sh);
                }
                __syncthreads();                                                  // row_max, row_log, best
                if (tid < lim && (tid < found || tid < p.k)) {
                    uint32_t rank = tid;
                    uint64_t rec = ~0ull;
                    if (tid < found) {
                        rec = sh.best[tid];
                        rank = 0;
                        for (uint32_t i = 0; i < found; ++i) rank += sh.best[i] < rec;
                    }
                    if (rank < p.k) {
                        float lp = NAN;                                           // fewer than k elements that are no NaN
                        int64_t token = -1;
                        if (rec != ~0ull) {
                            const float x = __uint_as_float(bits32_from_key(record_key(rec)));
                            const float log_s = sh.row_log;
                            lp = log_s == -INFINITY ? -INFINITY : (x - sh.row_max) * p.scale - log_s;
                            token = (int64_t)record_idx(rec);
                        }
                        p.top_logprobs[row * p.k + rank] = lp;
                        p.top_tokens[row * p.k + rank] = token;
                    }
                }
            }
        }
        turn ^= 1;
        __syncthreads();
    }
    lp_cp_wait<0>();
    if (parts > 1) cluster.sync();                                                // no CTA leaves while its memory is written
}

// ---------------------------------------------------------------------------------------------------------------------
// Gradient.  With upstream gradients g_lp (of the token's log probability), g_H, g_lse and g_j (of the alternatives'),
//   dL/dx_v = (1/T) [ -p_v (G + g_H (ln p_v + H)) + g_lp 1[v = token] + sum_j g_j 1[v = i_j] ],   G = g_lp + sum_j g_j - g_lse,
// p_v = e^(x_v / T - lse): one read and one write of the matrix; the picked entries are written again behind a barrier.
struct LpGradParams {
    const void* logits;
    void* grad;
    int64_t rows, row_stride, grad_stride;
    uint32_t V, k, chunks;               // chunks per row
    uint32_t chunk;                      // elements per chunk
    float scale;
    const int64_t* tokens;               // the pointers below may be null, except lse
    const float* lse;
    const float* lse_rest;
    const float* entropy;
    const float* g_logprob;
    const float* g_entropy;
    const float* g_lse;
    const int64_t* top_tokens;
    const float* g_top;
};

constexpr int LG_THREADS = 256;
constexpr int LG_UNROLL = 4;

struct LgRow { float lse, rest, whole, g_h; };      // lse in two floats; (G + g_H H) / T; g_H / T

__device__ __forceinline__ float lg_dense(float x, const LgRow& r, float scale) {
    const float a = fmaf(x, scale, -r.lse) - r.rest;
    const float q = exp2_approx(a * LOG2E);
    return -q * fmaf(r.g_h, fmaxf(a, FAR_BELOW), r.whole);
}

template <typename T>
__global__ void __launch_bounds__(LG_THREADS) logprobs_grad_kernel(const LpGradParams p) {
    constexpr int VEC = Logit<T>::VEC, U = LG_UNROLL;
    __shared__ float s_sum[LG_THREADS / 32];
    const unsigned tid = threadIdx.x;
    const int64_t row = blockIdx.x / p.chunks;
    const uint32_t chunk = (uint32_t)(blockIdx.x % p.chunks);
    pdl_wait();
    pdl_launch_dependents();
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.row_stride;
    T* y = reinterpret_cast<T*>(p.grad) + row * p.grad_stride;
    const int64_t token = p.tokens ? p.tokens[row] : -1;
    const bool given = token >= 0 && token < (int64_t)p.V;
    const float g_lp = p.g_logprob && given ? p.g_logprob[row] : 0.f;
    const float scale = p.scale;
    float g_sum = 0.f;
    if (p.g_top) {
        float g = 0.f;
        for (uint32_t j = tid; j < p.k; j += LG_THREADS) g += p.g_top[row * p.k + j];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) g += __shfl_xor_sync(FULL_MASK, g, d);
        if ((tid & 31) == 0) s_sum[tid >> 5] = g;
        __syncthreads();
        for (int w = 0; w < LG_THREADS / 32; ++w) g_sum += s_sum[w];
    }
    LgRow r;
    r.lse = p.lse[row];
    r.rest = p.lse_rest ? p.lse_rest[row] : 0.f;
    const float g_h = p.g_entropy ? p.g_entropy[row] : 0.f;
    const float whole = g_lp + g_sum - (p.g_lse ? p.g_lse[row] : 0.f);
    r.whole = (whole + (p.g_entropy ? g_h * p.entropy[row] : 0.f)) * scale;
    r.g_h = g_h * scale;
    const bool empty = r.lse == -INFINITY;                 // nothing but -inf in the row: no gradient

    const uint32_t e0 = chunk * p.chunk, e1 = min(p.V, e0 + p.chunk);
    const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(x + e0) & 15u);
    const bool aligned = mis == (uint32_t)(reinterpret_cast<uintptr_t>(y + e0) & 15u);
    auto scalar = [&](uint32_t i) { y[i] = Logit<T>::from_float(empty ? 0.f : lg_dense(Logit<T>::to_float(x[i]), r, scale)); };
    if (aligned) {
        const uint32_t head = min(e1, e0 + (mis ? (16u - mis) / (uint32_t)sizeof(T) : 0u));
        const uint32_t nvec = (e1 - head) / VEC, tail = head + nvec * VEC;
        if (e0 + tid < head) scalar(e0 + tid);
        if (tail + tid < e1) scalar(tail + tid);
        for (uint32_t v = tid; v < nvec; v += LG_THREADS * U) {
            uint4 in[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * LG_THREADS < nvec) in[u] = ld_stream_u4(x + head + (size_t)(v + u * LG_THREADS) * VEC);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * LG_THREADS < nvec) {
                    float f[VEC];
                    Logit<T>::unpack(in[u], f);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) f[j] = empty ? 0.f : lg_dense(f[j], r, scale);
                    st_stream_u4(y + head + (size_t)(v + u * LG_THREADS) * VEC, Logit<T>::pack(f));
                }
            }
        }
    } else {                                               // gradient rows that start at another offset than the logits'
        for (uint32_t i = e0 + tid; i < e1; i += LG_THREADS) scalar(i);
    }
    if (empty || (!given && !p.g_top)) return;
    __syncthreads();
    // the picked entries of this chunk: everything that falls on one of them is summed before it is rounded
    for (uint32_t j = tid; j <= p.k; j += LG_THREADS) {
        const int64_t i = j < p.k ? (p.g_top ? p.top_tokens[row * p.k + j] : -1) : (given ? token : -1);
        if (i < (int64_t)e0 || i >= (int64_t)e1) continue;
        float g = i == token ? g_lp : 0.f;
        if (p.g_top)
            for (uint32_t q = 0; q < p.k; ++q) g += p.top_tokens[row * p.k + q] == i ? p.g_top[row * p.k + q] : 0.f;
        y[i] = Logit<T>::from_float(fmaf(g, scale, lg_dense(Logit<T>::to_float(x[i]), r, scale)));
    }
}

}  // namespace profk
