// Log probabilities of given tokens, entropy and top alternatives of every row of a logits matrix, in one read of it,
// and their gradient.
//
// With z = x / T, a reference m and s = sum e^(z - m) over a row:   lse = m + ln s,   ln p_v = z_v - lse,
//   H = -sum p ln p = ln s - (1/s) sum e^(z - m) (z - m).
// A part of a row is described by (mx, s, t), m = mx / T and t = sum e^(z - m) (x - mx), with mx a logit of the row that none
// of the part exceeds; two parts join by moving both to the larger mx, so every thread keeps a triple of its own and they are
// joined in a fixed order at the end of the row.  In the end mx is the row's largest logit, whose own term is 1 exactly: s >= 1
// and t <= 0, so that no log probability is above 0 and no entropy below, however sure the model is.  (A reference that lagged
// by up to 2^32 and moved less often takes 1 % off the time of scoring, and 1e-6 of accuracy.)  T only enters as a factor of the
// exponent: e^(z - m) = 2^((x - mx) log2(e) / T).
//
// What bounds it: fp32 the stream from HBM (1184 rows of 131072: 98 us, 6.3 TB/s without alternatives, 6.1 with five); 16-bit
// types have twice the exponentials per byte, and without alternatives the unit that takes them (16 per SM and cycle) is 70 %
// busy (2368 rows of bf16: 105 us, 5.9 TB/s), the issue slots as much, whence the packed arithmetic, the one look per batch and
// thread, and everything rare out of the way.  With five alternatives the same rows take 135 us, with twenty 168, and nothing is
// saturated (unit 52 %, issue slots 65 %, DRAM 51 %): the warps wait for the barrier of each row's first bound, and notes.  Steps
// on the way for five: a barrier and a look at every element per batch 254 us, notes 158, one CTA per SM 154, one look per batch
// 142, no 64-bit divisions 139, half warps' slots 137.
//
// The k largest logits are found on the way.  Groups of lanes keep the largest logit that they have seen in a slot of
// shared memory; the k-th largest slot is a bound that k elements of the row reach, so that only vectors whose maximum
// reaches the bound can matter.  Their numbers are noted in a list, a few times k of them for a row in any ordinary order;
// the bound is renewed whenever the number of batches has doubled, without a barrier: a stale slot only makes it lower.
// At the end of the row those that still matter are read once more and their elements above the last bound are ordered.  Where
// the list overflows all the same (ascending order, a flood of equal values, a hundred alternatives of a million tokens) the whole
// row is read once more instead, by one warp, while the others wait: right, and slow (2368 rows of bf16 with five: 870 us where all
// values are equal, 3000 in ascending order; 592 rows of 1048576 with 128: 945, with five 236).
//
// A CTA holds the whole SM and is two teams of twelve warps, each with rows of its own (or a part of a row each).  Eleven
// warps of a team stream; the first, which the scheduler prefers, finishes rows (joins the statistics, orders the list,
// writes the results) while the others are in the next one.  The teams' warps alternate in age: as two CTAs of an SM, one
// of them finished a third earlier than the other (89 us against 124) and left the SM half idle.
#pragma once

#include <cooperative_groups.h>

#include <type_traits>

#include "logits.cuh"

namespace profk {

namespace cg = cooperative_groups;

constexpr int LP_TEAMS = 2;
constexpr int LP_STREAM_WARPS = 11;
constexpr int LP_TEAM = (LP_STREAM_WARPS + 1) * 32;     // threads of a team
constexpr int LP_STREAM = LP_STREAM_WARPS * 32;
constexpr int LP_THREADS = LP_TEAMS * LP_TEAM;
constexpr int LP_UNROLL = 4;              // 16-byte vectors per thread and batch
constexpr int LP_STAGES = 3;              // batches in flight or in hand per thread
constexpr uint32_t LP_STEP = LP_STREAM * LP_UNROLL;     // vectors per batch
constexpr uint32_t LP_NOTES = 2560;       // vectors the list holds (k = 128 of 131072 fp32, normal: 1570 on average, 2420 at most in 1184 rows)
constexpr uint32_t LP_READ = 128;         // ... of which the finishing warp reads so many at a time
constexpr uint32_t LP_FIN = 512;          // elements the finishing warp holds; more than half of them it cuts back
constexpr uint32_t LP_MAX_K = 128;        // most alternatives
constexpr uint32_t LP_MAX_PARTS = 16;     // most teams that share a row
constexpr uint32_t LP_SLACK = 32;         // a part of a row hands on up to k + LP_SLACK records

struct LpParams {
    const void* logits;
    int64_t rows, row_stride;
    uint32_t V, k;
    uint32_t parts, parts_log2;           // teams that share a row: 1, or twice the CTAs of a cluster (a power of two)
    float scale, unscale;                 // 1 / T, and its reciprocal
    const int64_t* tokens;                // may be null
    float* logprob;
    float* lse;
    float* lse_rest;                      // may be null
    float* entropy;
    float* top_logprobs;
    int64_t* top_tokens;
};

struct LpStats { float m, s, t; };

// lse in two floats.  `near` is its rounding, `rest` what that left off.  From 2^30 on that would be two things, the rounding of
// max / T and ln s, and a float that holds the first (2^-24 of max / T) has no place for the second.  There rest is ln s, and its
// last three bits say which float around near T the row's largest logit is (as many floats on as these bits, less 3), from which
// the gradient then takes the exponents.  near T is off by three roundings and ln s, which is 3 floats at most.
constexpr float LP_HUGE = 1073741824.f;
__device__ __forceinline__ float lp_rest(float near, float m, float log_s, float scale, float unscale) {
    if (isinf(near)) return 0.f;
    if (!(fabsf(near) >= LP_HUGE)) return fmaf(m, scale, -near) + log_s;
    const int on = __float_as_int(m) - __float_as_int(near * unscale);
    return __int_as_float((__float_as_int(log_s) & ~7) | (min(max(on, -3), 3) + 3));
}
__device__ __forceinline__ float lp_max_of(float near, float rest, float unscale) {
    return __int_as_float(__float_as_int(near * unscale) + (__float_as_int(rest) & 7) - 3);
}

// Both parts moved to the larger maximum; c = log2(e) / T.
__device__ __forceinline__ LpStats lp_join(const LpStats& a, const LpStats& b, float c) {
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf(a.m - m, FAR_BELOW), db = fmaxf(b.m - m, FAR_BELOW);
    const float fa = exp2_approx(da * c), fb = exp2_approx(db * c);
    return LpStats{m, fa * a.s + fb * b.s, fa * fmaf(da, a.s, a.t) + fb * fmaf(db, b.s, b.t)};
}

// Bits that the number of any of the row's vectors takes.
template <typename T> __device__ __forceinline__ uint32_t lp_note_bits(uint32_t V) { return 32 - __clz(V / Logit<T>::VEC | 1); }

// What the streaming warps leave of a row for the finishing one; two of them, used in turn.
struct LpRow {
    uint32_t note[LP_NOTES];              // vectors: numbers in the low `lp_note_bits`, above them the head of the largest element's order key
    LpStats stats[LP_STREAM_WARPS];
    uint32_t count;
    float bound;                          // elements below it are no longer of interest
};

struct LpShared {
    LpRow row[2];
    uint64_t fin[LP_FIN];                 // records, of the finishing warp
    float slot[LP_STREAM];                // largest logits seen by a group of lanes
    float half[LP_STREAM / 16];           // ... by half a warp
};

// Named barriers of a team: among its streaming warps; a row is ready for the finishing warp; its place may be used again.
struct LpBarriers {
    int base;
    __device__ __forceinline__ explicit LpBarriers(int team) : base(1 + 5 * team) {}
    __device__ __forceinline__ void full_arrive(int turn) const { asm volatile("bar.arrive %0, %1;" ::"r"(base + 1 + turn), "n"(LP_TEAM) : "memory"); }
    __device__ __forceinline__ void full_sync(int turn) const { asm volatile("bar.sync %0, %1;" ::"r"(base + 1 + turn), "n"(LP_TEAM) : "memory"); }
    __device__ __forceinline__ void empty_arrive(int turn) const { asm volatile("bar.arrive %0, %1;" ::"r"(base + 3 + turn), "n"(LP_TEAM) : "memory"); }
    __device__ __forceinline__ void empty_sync(int turn) const { asm volatile("bar.sync %0, %1;" ::"r"(base + 3 + turn), "n"(LP_TEAM) : "memory"); }
    // How many of the streaming threads say yes.
    __device__ __forceinline__ uint32_t count(bool yes) const {
        uint32_t n;
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.popc.u32 %0, %2, %3, p;\n\t}"
                     : "=r"(n) : "r"((uint32_t)yes), "r"(base), "n"(LP_STREAM) : "memory");
        return n;
    }
};

// By one warp: a limit (found by halving the interval of the records' value words, then of their index words) such that
// at least k and at most `most` of the n records in `a` are <= it; no more than `most` valid records (~0 is none): all of
// them.  A warp barrier must lie between the last write to `a` and the call.
__device__ __forceinline__ uint64_t lp_find_limit(const uint64_t* a, uint32_t n, uint32_t k, uint32_t most) {
    uint32_t lo = 0xFFFFFFFFu, hi = 0u, valid = 0;
    for (uint32_t i = lane_id(); i < n; i += 32) {
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
    if (__reduce_add_sync(FULL_MASK, valid) <= most) return ~0ull - 1;
    // smallest value word `lo` with at least k records at or below it (a ~0 record lies above every limit used)
    while (lo < hi) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        uint32_t c = 0;
#pragma unroll 4
        for (uint32_t i = lane_id(); i < n; i += 32) c += (uint32_t)(a[i] >> 32) <= mid;
        c = __reduce_add_sync(FULL_MASK, c);
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
        for (uint32_t i = lane_id(); i < n; i += 32) c += a[i] <= limit;
        c = __reduce_add_sync(FULL_MASK, c);
        if (c >= k) {
            ihi = mid;
            if (c <= most) break;
        } else {
            ilo = mid + 1;
        }
    }
    return ((uint64_t)word << 32) | ihi;
}

// Lanes that share a slot: the coarser the slots the cheaper the bound, the finer the tighter (the k-th largest of n slots
// has about n ln(n / (n - k)) elements above it).
constexpr uint32_t LP_RANKED = LP_MAX_K + LP_SLACK;     // records that are ranked against one another
// Up to here 22 slots, one per lane of a warp, whose k-th largest is found by counting: 2368 rows of 131072 bf16, k = 8: 135 us,
// with the bisection over all threads that larger k take 154; 4 rows, k = 16: 11.2 against 12.9.
constexpr uint32_t LP_FEW_K = 16;
__device__ __forceinline__ uint32_t lp_slot_lanes(uint32_t k) { return k <= LP_FEW_K ? 16 : k <= 64 ? 4 : 1; }

// Both kinds of slots; the coarser ones serve alone for few alternatives (slot_lanes 16).
__device__ __forceinline__ void lp_write_slot(float seen, uint32_t tid, uint32_t lanes, LpShared& sh) {
    if (lanes == 1) sh.slot[tid] = seen;
    seen = fmaxf(seen, __shfl_xor_sync(FULL_MASK, seen, 1));
    seen = fmaxf(seen, __shfl_xor_sync(FULL_MASK, seen, 2));
    if (lanes == 4 && (tid & 3) == 0) sh.slot[tid / 4] = seen;
    seen = fmaxf(seen, __shfl_xor_sync(FULL_MASK, seen, 4));
    seen = fmaxf(seen, __shfl_xor_sync(FULL_MASK, seen, 8));
    if ((tid & 15) == 0) sh.half[tid / 16] = seen;
}

// A count that is near enough: at least k values reach the bound, and not many more.
__device__ __forceinline__ uint32_t lp_enough(uint32_t k) { return k + k / 8 + 1; }

// By any warp: the k-th largest of the half warps' slots, k <= LP_FEW_K, by counting.
__device__ __forceinline__ float lp_half_bound(uint32_t k, const LpShared& sh) {
    constexpr uint32_t N = LP_STREAM / 16;
    const uint32_t lane = lane_id();
    const volatile float* slot = sh.half;
    const float mine = lane < N ? slot[lane] : -INFINITY;
    uint32_t above = 0;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) above += __shfl_sync(FULL_MASK, mine, i) > mine;
    // of the slots with fewer than k larger ones the smallest: at least k slots reach it
    const uint32_t key = above < k && lane < N ? key_from_bits32(float_bits_exact(mine)) : 0xFFFFFFFFu;
    return __uint_as_float(bits32_from_key(__reduce_min_sync(FULL_MASK, key)));
}

// By one warp: a bound from the slots that is no lower than `bound`.
__device__ __forceinline__ float lp_slot_bound(float bound, uint32_t k, uint32_t lanes, const LpShared& sh) {
    if (lanes == 16) return fmaxf(bound, lp_half_bound(k, sh));
    const uint32_t n = LP_STREAM / lanes, lane = lane_id();
    const volatile float* slot = sh.slot;
    uint32_t top = 0, reach = 0;
    uint32_t lo = key_from_bits32(float_bits_exact(bound));
    for (uint32_t at = lane; at < n; at += 32) {
        const uint32_t key = key_from_bits32(float_bits_exact(slot[at]));
        top = max(top, key);
        reach += key >= lo;
    }
    if (__reduce_add_sync(FULL_MASK, reach) < k) return bound;                    // (slots of groups: coarser than the first bound)
    uint32_t hi = __reduce_max_sync(FULL_MASK, top) + 1u;
    while (lo + 1 < hi) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        uint32_t c = 0;                                                           // (a slot that rises meanwhile does no harm)
#pragma unroll 4
        for (uint32_t at = lane; at < n; at += 32) c += key_from_bits32(float_bits_exact(slot[at])) >= mid;
        c = __reduce_add_sync(FULL_MASK, c);
        if (c >= k) {
            lo = mid;
            if (c <= lp_enough(k)) break;
        } else {
            hi = mid;
        }
    }
    return __uint_as_float(bits32_from_key(lo));
}

// By the streaming warps: (nearly) the k-th largest of the logits `seen` by their threads: of half warps' for few, else by
// halving the interval of their order keys.  They are LOWEST at least, and so is the bound: -inf is never noted on the
// way.  The slots must be written; a barrier lies within.
__device__ __forceinline__ float lp_first_bound(float seen, uint32_t k, LpShared& sh, const LpBarriers& bar) {
    if (k <= LP_FEW_K) {
        bar.count(true);
        return lp_half_bound(k, sh);
    }
    const uint32_t key = key_from_bits32(float_bits_exact(seen));
    uint32_t lo = key_from_bits32(0xFF7FFFFFu), hi = key_from_bits32(0x7F800000u) + 1u;
    while (lo + 1 < hi) {
        const uint32_t mid = lo + ((hi - lo) >> 1), c = bar.count(key >= mid);
        if (c >= k) {
            lo = mid;
            if (c <= lp_enough(k)) break;
        } else {
            hi = mid;
        }
    }
    return __uint_as_float(bits32_from_key(lo));
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
    __device__ __forceinline__ void set(const LpParams& p, int64_t row, uint32_t part) {
        x = reinterpret_cast<const T*>(p.logits) + row * p.row_stride;
        const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(x) & 15u);
        head = min(p.V, mis ? (16u - mis) / (uint32_t)sizeof(T) : 0u);
        nvec = (p.V - head) / Logit<T>::VEC;
        v0 = (uint32_t)((uint64_t)nvec * part >> p.parts_log2);
        v1 = (uint32_t)((uint64_t)nvec * (part + 1) >> p.parts_log2);
    }
    __device__ __forceinline__ const T* vec(uint32_t v) const { return x + head + (size_t)v * Logit<T>::VEC; }
};

// ---- the finishing warp's part of a selection; `n` records are in sh.fin, all lanes agree on it

// Drops the records above `limit`; keeps the others' order.
__device__ __forceinline__ uint32_t lp_fin_drop(uint32_t n, uint64_t limit, LpShared& sh) {
    uint32_t kept = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += 32) {
        const uint64_t r = i0 + lane_id() < n ? sh.fin[i0 + lane_id()] : ~0ull;
        __syncwarp();
        const bool keep = r <= limit && r != ~0ull;
        const unsigned who = __ballot_sync(FULL_MASK, keep);
        if (keep) sh.fin[kept + __popc(who & ((1u << lane_id()) - 1u))] = r;
        kept += __popc(who);
        __syncwarp();
    }
    return kept;
}
// Adds each lane's element if it has one (lp_fin_vector leaves room for it).
__device__ __forceinline__ uint32_t lp_fin_add(uint32_t n, bool has, float x, uint32_t idx, LpShared& sh) {
    const unsigned who = __ballot_sync(FULL_MASK, has);
    if (who == 0) return n;
    if (has) sh.fin[n + __popc(who & ((1u << lane_id()) - 1u))] = make_record(key_from_bits32(float_bits_exact(x)), idx);
    __syncwarp();
    return n + __popc(who);
}
// The elements of one vector per lane (`has`) that reach the bound; cuts back to the k best and some before the room runs out,
// and then raises the bound above the worst of them where what follows has higher indices only (`ascending`).
template <typename T>
__device__ __forceinline__ uint32_t lp_fin_vector(uint32_t n, bool has, const uint4& vec, uint32_t at, float& bound, bool ascending, uint32_t k, LpShared& sh) {
    has = has && Logit<T>::vec_max(vec) >= bound;
    if (!__any_sync(FULL_MASK, has)) return n;
    float x[Logit<T>::VEC];
    Logit<T>::unpack(vec, x);
    uint32_t hits = 0;
#pragma unroll
    for (int j = 0; j < Logit<T>::VEC; ++j) hits |= (has && x[j] >= bound ? 1u : 0u) << j;
    uint32_t incl = __popc(hits);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t up = __shfl_up_sync(FULL_MASK, incl, d);
        if (lane_id() >= (uint32_t)d) incl += up;
    }
    uint32_t pos = n + incl - __popc(hits);
#pragma unroll
    for (int j = 0; j < Logit<T>::VEC; ++j)
        if (hits >> j & 1) sh.fin[pos++] = make_record(key_from_bits32(float_bits_exact(x[j])), at + j);
    n += __shfl_sync(FULL_MASK, incl, 31);
    __syncwarp();
    if (n > LP_FIN / 2) {
        const uint64_t limit = lp_find_limit(sh.fin, n, k, LP_RANKED);
        n = lp_fin_drop(n, limit, sh);
        if (ascending) bound = __uint_as_float(bits32_from_key(~(uint32_t)(limit >> 32) + 1u));
    }
    return n;
}

// Drops the notes of vectors that cannot matter, most of them from the start of the row when the bound was low: the k-th largest
// of the noted vectors' largest elements, rounded down to the bits that a note has of them, is a bound of its own.  Returns how many
// remain.  (What is left out costs a read by latency each: k = 128 of 131072, 2368 rows bf16 329 -> 216 us, 1184 rows fp32
// 371 -> 141 to 171; fewer notes than LP_READ are read at once, 1981 rows of 5946 bf16, k = 64: 48 us, thinned 56.)
__device__ __forceinline__ uint32_t lp_fin_thin(uint32_t notes, uint32_t k, uint32_t bits, float& bound, LpRow& r) {
    uint32_t top = 0;
    for (uint32_t i = lane_id(); i < notes; i += 32) top = max(top, r.note[i] >> bits);
    uint32_t lo = key_from_bits32(float_bits_exact(bound)) >> bits, hi = __reduce_max_sync(FULL_MASK, top) + 1u;
    while (lo + 1 < hi) {                                                         // (the first `lo` is the bound of the slots)
        const uint32_t mid = (lo + hi) >> 1;
        uint32_t c = 0;
#pragma unroll 4
        for (uint32_t i = lane_id(); i < notes; i += 32) c += r.note[i] >> bits >= mid;
        c = __reduce_add_sync(FULL_MASK, c);
        if (c >= k) {
            lo = mid;
            if (c <= lp_enough(k)) break;
        } else {
            hi = mid;
        }
    }
    bound = fmaxf(bound, __uint_as_float(bits32_from_key(lo << bits)));
    uint32_t kept = 0;
    for (uint32_t i0 = 0; i0 < notes; i0 += 32) {
        const uint32_t i = i0 + lane_id();
        const uint32_t w = i < notes ? r.note[i] : 0u;
        const bool keep = i < notes && w >> bits >= lo;
        const unsigned who = __ballot_sync(FULL_MASK, keep);
        if (keep) r.note[kept + __popc(who & ((1u << lane_id()) - 1u))] = w;      // (at or before i0 + lane: read already)
        kept += __popc(who);
        __syncwarp();
    }
    return kept;
}

// The candidates of a row's share, at most `most` (>= k) of them, the k best of the row among them as far as they lie here.
template <typename T>
__device__ __forceinline__ uint32_t lp_fin_select(const LpShare<T> mine, uint32_t k, uint32_t most, bool first, bool last, uint32_t V, LpRow& r, LpShared& sh) {
    constexpr int VEC = Logit<T>::VEC;
    const uint32_t lane = lane_id();
    uint32_t n = 0;
    float bound = r.bound;
    uint32_t notes = r.count;
    const uint32_t bits = lp_note_bits<T>(V);
    const uint32_t tail = mine.head + mine.nvec * VEC;
    const bool in_head = first && lane < mine.head, in_tail = last && tail + lane < V;
    const float hx = in_head ? Logit<T>::to_float(mine.x[lane]) : -INFINITY, tx = in_tail ? Logit<T>::to_float(mine.x[tail + lane]) : -INFINITY;
    n = lp_fin_add(n, hx >= bound, hx, lane, sh);
    if (notes <= LP_NOTES) {
        if (notes > LP_READ && notes >= k) notes = lp_fin_thin(notes, k, bits, bound, r);
        for (uint32_t i0 = 0; i0 < notes; i0 += LP_READ) {
            uint32_t w[4];
            uint4 vec[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t i = i0 + u * 32 + lane;
                w[u] = i < notes ? r.note[i] & ((1u << bits) - 1u) : 0u;
                if (i < notes) vec[u] = *reinterpret_cast<const uint4*>(mine.vec(w[u]));
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i0 + u * 32 < notes) n = lp_fin_vector<T>(n, i0 + u * 32 + lane < notes, vec[u], mine.head + w[u] * VEC, bound, false, k, sh);
        }
    } else {
        for (uint32_t v = mine.v0; v < mine.v1; v += 128) {
            uint4 vec[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (v + u * 32 + lane < mine.v1) vec[u] = ld_stream_u4(mine.vec(v + u * 32 + lane));
#pragma unroll
            for (int u = 0; u < 4; ++u)
                n = lp_fin_vector<T>(n, v + u * 32 + lane < mine.v1, vec[u], mine.head + (v + u * 32 + lane) * VEC, bound, true, k, sh);
        }
    }
    n = lp_fin_add(n, tx >= bound, tx, tail + lane, sh);
    // Masked tokens (-inf) fill the places that nothing else takes, lowest indices first.  (A bound above LOWEST says that
    // the row has k others; of a part it may have fewer.)
    const bool short_of = r.bound == LOWEST;
    const uint32_t e1 = last ? V : mine.head + mine.v1 * VEC;
    for (uint32_t e = (first ? 0 : mine.head + mine.v0 * VEC); short_of && n < k && e < e1; e += 32)
        n = lp_fin_add(n, e + lane < e1 && Logit<T>::to_float(mine.x[e + lane]) == -INFINITY, -INFINITY, e + lane, sh);
    if (n > most) n = lp_fin_drop(n, lp_find_limit(sh.fin, n, k, most), sh);
    return n;
}

struct LpTeamMemory {
    uint4 ring[LP_STAGES * LP_STEP];
    LpShared sh;
};

// A team takes a row at a time (parts = 1), or the teams of a cluster of CTAs a part of a row each.  The vectors of
// the row come through a ring in shared memory that each thread fills and empties for itself (cp.async, no barrier), and
// that runs on into the next row, so that HBM stays busy while a row is finished.
template <typename T, bool ENT, bool TOPK>
__global__ void __launch_bounds__(LP_THREADS, 1) logprobs_kernel(const LpParams p) {
    constexpr int VEC = Logit<T>::VEC, U = LP_UNROLL;
    extern __shared__ __align__(16) unsigned char lp_dyn[];
    const uint32_t lane = lane_id(), cta_warp = threadIdx.x >> 5;
    const int team = (cta_warp >> 2) & 1;
    const int warp = (int)((cta_warp >> 3) * 4 + (cta_warp & 3)) - 1;              // of the team: -1 finishes, 0 .. stream
    const uint32_t tid = warp * 32 + lane;
    LpTeamMemory& mem = reinterpret_cast<LpTeamMemory*>(lp_dyn)[team];
    LpShared& sh = mem.sh;
    const uint4* ring = mem.ring;                                                 // [LP_STAGES][U][LP_STREAM]
    const LpBarriers bar(team);
    const uint32_t lim = TOPK ? p.k + LP_SLACK : 0;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t parts = p.parts, part = parts > 1 ? cluster.block_rank() * LP_TEAMS + team : 0;
    // what the parts of a row hand to the first of them: two sets, used in turn
    uint64_t* in_recs = reinterpret_cast<uint64_t*>(lp_dyn + LP_TEAMS * sizeof(LpTeamMemory));              // [2][parts * lim]
    LpStats* in_stats = reinterpret_cast<LpStats*>(in_recs + 2 * (size_t)parts * lim);                     // [2][parts]
    float* in_bounds = reinterpret_cast<float*>(in_stats + 2 * parts);                                     // [2][2][parts], in every CTA
    __shared__ uint32_t in_found[2];                                              // records in the list
    if (threadIdx.x < 2) in_found[threadIdx.x] = 0;
    if (parts > 1) __syncthreads();

    const uint32_t shares = parts > 1 ? parts / LP_TEAMS : 1;                     // CTAs per row
    const int32_t rows = (int32_t)p.rows;
    const int32_t first = parts > 1 ? (int32_t)(blockIdx.x / shares) : (int32_t)(blockIdx.x * LP_TEAMS + team);
    const int32_t stride = parts > 1 ? (int32_t)(gridDim.x / shares) : (int32_t)(gridDim.x * LP_TEAMS);
    auto row_after = [&](int32_t row) { return row > rows - stride ? rows : row + stride; };     // (rows may be 2^31 - 1: row + stride would wrap)
    const float c = p.scale * LOG2E;
    pdl_wait();
    pdl_launch_dependents();
    if (parts > 1) cluster.sync();                                                // every CTA of the cluster has started

    int turn = 0;
    if (warp < 0) {
        // ---- the finishing warp
        auto make_empty = [&](int t) {
            if (lane == 0) { sh.row[t].count = 0; sh.row[t].bound = LOWEST; }
            __syncwarp();
            bar.empty_arrive(t);
        };
        if (first < rows) make_empty(0);
        if (stride < rows - first) make_empty(1);
        for (int32_t row = first; row < rows; row = row_after(row)) {
            const int64_t token = p.tokens ? p.tokens[row] : -1;
            float token_x = 0.f;
            if (token >= 0 && token < (int64_t)p.V) token_x = Logit<T>::to_float((reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.row_stride)[token]);
            if constexpr (TOPK)
                if (parts > 1) {                                                  // the streaming warps exchange bounds, see there
                    cluster.sync();
                    if (__any_sync(FULL_MASK, lane < parts && in_bounds[turn * 2 * parts + lane] == LOWEST)) cluster.sync();
                }
            bar.full_sync(turn);
            LpRow& r = sh.row[turn];
            // join the warps' statistics, in a fixed order; every lane gets the result
            auto join_lanes = [&](LpStats st, int width) {
                for (int d = width / 2; d > 0; d >>= 1) {
                    LpStats o;
                    o.m = __shfl_xor_sync(FULL_MASK, st.m, d);
                    o.s = __shfl_xor_sync(FULL_MASK, st.s, d);
                    o.t = __shfl_xor_sync(FULL_MASK, st.t, d);
                    st = (lane & d) ? lp_join(o, st, c) : lp_join(st, o, c);
                }
                return st;
            };
            LpStats all = join_lanes(lane % 16 < LP_STREAM_WARPS ? r.stats[lane % 16] : LpStats{LOWEST, 0.f, 0.f}, 16);
            uint32_t found = 0;
            if constexpr (TOPK) {
                LpShare<T> mine;
                mine.set(p, row, part);
                found = lp_fin_select<T>(mine, p.k, parts > 1 ? lim : LP_RANKED, part == 0, part == parts - 1, p.V, r, sh);
            }
            if (parts > 1) {
                // hand statistics and records to the cluster's first CTA
                if constexpr (TOPK) {
                    uint32_t at = 0;
                    if (lane == 0 && found > 0) at = atomicAdd(cluster.map_shared_rank(in_found, 0) + turn, found);
                    at = __shfl_sync(FULL_MASK, at, 0);
                    uint64_t* to_recs = cluster.map_shared_rank(in_recs, 0) + (size_t)turn * parts * lim + at;
                    for (uint32_t i = lane; i < found; i += 32) to_recs[i] = sh.fin[i];
                }
                if (lane == 0) *(cluster.map_shared_rank(in_stats, 0) + turn * parts + part) = all;
                __syncwarp();
                cluster.sync();
                if (part == 0) {
                    all = join_lanes(lane % 16 < parts ? in_stats[turn * parts + lane % 16] : LpStats{LOWEST, 0.f, 0.f}, 16);
                    if constexpr (TOPK) {
                        const uint64_t* recs = in_recs + (size_t)turn * parts * lim;
                        const uint32_t n = in_found[turn];
                        const uint64_t limit = n > LP_RANKED ? lp_find_limit(recs, n, p.k, LP_RANKED) : ~0ull;
                        found = 0;
                        for (uint32_t i0 = 0; i0 < n; i0 += 32) {
                            const bool keep = i0 + lane < n && recs[i0 + lane] <= limit;
                            const unsigned who = __ballot_sync(FULL_MASK, keep);
                            if (keep) sh.fin[found + __popc(who & ((1u << lane) - 1u))] = recs[i0 + lane];
                            found += __popc(who);
                        }
                        __syncwarp();
                        if (lane == 0) in_found[turn] = 0;
                    }
                }
            }
            if (part == 0) {
                const bool empty = all.s == 0.f;                                  // nothing but -inf
                const float log_s = logf(all.s);
                if (lane == 0) {
                    // lse in two floats: one alone loses ln s beside a large maximum (all of it in a row masked with fp32's
                    // lowest value), and with it the probabilities that the gradient takes from it
                    const float near = empty ? -INFINITY : fmaf(all.m, p.scale, log_s);
                    p.lse[row] = near;
                    if (p.lse_rest) p.lse_rest[row] = lp_rest(near, all.m, log_s, p.scale, p.unscale);
                    if constexpr (ENT) p.entropy[row] = empty ? 0.f : log_s - p.scale * (all.t / all.s);
                    if (p.logprob) {
                        float lp = 0.f;                                           // no token given
                        if (token >= (int64_t)p.V) lp = NAN;
                        else if (token >= 0) lp = empty ? -INFINITY : (token_x - all.m) * p.scale - log_s;
                        p.logprob[row] = lp;
                    }
                }
                if constexpr (TOPK) {
                    auto rank_and_write = [&](auto regs) {
                        constexpr int PER = decltype(regs)::value;                // records per lane
                        uint64_t rec[PER];
                        uint32_t rank[PER];
#pragma unroll
                        for (int i = 0; i < PER; ++i) {
                            const uint32_t at = i * 32 + lane;
                            rec[i] = at < found ? sh.fin[at] : ~0ull;
                            rank[i] = at < found ? 0 : at - found;                // (behind all that are valid)
                        }
#pragma unroll 4
                        for (uint32_t q = 0; q < found; ++q) {
                            const uint64_t other = sh.fin[q];
#pragma unroll
                            for (int i = 0; i < PER; ++i) rank[i] += other < rec[i];
                        }
#pragma unroll
                        for (int i = 0; i < PER; ++i) {
                            if (rank[i] >= p.k) continue;
                            float lp = NAN;                                       // fewer than k elements that are no NaN
                            int64_t at = -1;
                            if (rec[i] != ~0ull) {
                                const float x = __uint_as_float(bits32_from_key(record_key(rec[i])));
                                lp = empty ? -INFINITY : (x - all.m) * p.scale - log_s;
                                at = (int64_t)record_idx(rec[i]);
                            }
                            p.top_logprobs[(int64_t)row * p.k + rank[i]] = lp;
                            p.top_tokens[(int64_t)row * p.k + rank[i]] = at;
                        }
                    };
                    const uint32_t places = max(found, p.k);
                    if (places <= 32) rank_and_write(std::integral_constant<int, 1>{});
                    else if (places <= 64) rank_and_write(std::integral_constant<int, 2>{});
                    else if (places <= 96) rank_and_write(std::integral_constant<int, 3>{});
                    else if (places <= 128) rank_and_write(std::integral_constant<int, 4>{});
                    else rank_and_write(std::integral_constant<int, LP_RANKED / 32>{});
                }
            }
            __syncwarp();
            if ((int64_t)row + 2 * (int64_t)stride < rows) make_empty(turn);
            turn ^= 1;
        }
    } else {
        // ---- the streaming warps: the loading side runs LP_STAGES - 1 batches ahead of the working side
        const uint32_t slot_lanes = TOPK ? lp_slot_lanes(p.k) : 1;
        const F32x2 c2 = f2_make(c, c);
        int32_t load_row = first;
        const T* load_at = nullptr;                                               // this thread's first vector of the next batch
        int32_t load_left = 0;                                                    // ... and how many the share still has behind it
        int load_stage = 0;
        auto load_from = [&]() {
            if (load_row >= rows) return;
            LpShare<T> ld;
            ld.set(p, load_row, part);
            load_at = ld.vec(ld.v0 + tid);
            load_left = (int32_t)(ld.v1 - ld.v0);
        };
        load_from();
        const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring) + tid * 16u;
        auto load_batch = [&]() {
            if (load_row < rows) {
                const uint32_t to = ring_addr + load_stage * (LP_STEP * 16u);
                if (load_left >= (int32_t)LP_STEP) {
#pragma unroll
                    for (int u = 0; u < U; ++u) lp_cp_async16(to + u * (LP_STREAM * 16u), load_at + u * (LP_STREAM * VEC));
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (u * LP_STREAM + (int)tid < load_left) lp_cp_async16(to + u * (LP_STREAM * 16u), load_at + u * (LP_STREAM * VEC));
                }
                load_at += LP_STEP * VEC;
                load_left -= (int32_t)LP_STEP;
                if (load_left <= 0) {
                    load_row = row_after(load_row);
                    load_from();
                }
            }
            lp_cp_commit();
            load_stage = load_stage + 1 == LP_STAGES ? 0 : load_stage + 1;
        };
#pragma unroll
        for (int s = 0; s < LP_STAGES - 1; ++s) load_batch();

        // The least (or the largest) of the parts' bounds; the finishing warps take part in the barrier.
        auto lp_exchange = [&](float mine, bool largest) {
            const uint32_t set = (turn * 2 + (largest ? 1 : 0)) * parts;
            if (tid < shares) cluster.map_shared_rank(in_bounds, tid)[set + part] = mine;
            __syncwarp();
            cluster.sync();
            float b = lane < parts ? in_bounds[set + lane] : largest ? LOWEST : INFINITY;
#pragma unroll
            for (int d = LP_MAX_PARTS / 2; d > 0; d >>= 1) {
                const float o = __shfl_xor_sync(FULL_MASK, b, d);
                b = largest ? fmaxf(b, o) : fminf(b, o);
            }
            return __shfl_sync(FULL_MASK, b, 0);
        };

        int stage = 0;
        for (int32_t row = first; row < rows; row = row_after(row)) {
            LpShare<T> mine;
            mine.set(p, row, part);
            LpRow& r = sh.row[turn];
            // m: what the exponents of this thread are taken relative to, the largest logit that its warp has seen (one
            // reference for a warp: a new maximum gets rare soon, and one thread's would be one of 32 times as many).
            float m = LOWEST, seen = LOWEST;
            F32x2 s2 = f2_make(0.f, 0.f), t2 = s2;                                // even and odd elements apart
            auto raise = [&](float to) {                                          // the running maximum, and s and t to it
                const float d = fmaxf(m - to, FAR_BELOW), f = exp2_approx(d * c);
                const F32x2 f2 = f2_make(f, f);
                if constexpr (ENT) t2 = f2_mul(f2, f2_fma(f2_make(d, d), s2, t2));
                s2 = f2_mul(f2, s2);
                m = to;
            };
            auto pair = [&](float a, float b, F32x2 minus_m, F32x2& s2, F32x2& t2) {        // (a masked element makes t NaN: 0 * -inf)
                const F32x2 d = f2_add(f2_make(a, b), minus_m);
                float ya, yb;
                f2_split(f2_mul(d, c2), ya, yb);
                const F32x2 e = f2_make(exp2_approx(ya), exp2_approx(yb));
                s2 = f2_add(s2, e);
                if constexpr (ENT) t2 = f2_fma(e, d, t2);
            };
            auto masked_pair = [&](float a, float b, F32x2 minus_m, F32x2& t2) {  // t alone, a masked element adds nothing to it
                float da, db;
                f2_split(f2_add(f2_make(a, b), minus_m), da, db);
                t2 = f2_fma(f2_make(exp2_approx(da * c), exp2_approx(db * c)), f2_make(fmaxf(da, FAR_BELOW), fmaxf(db, FAR_BELOW)), t2);
            };
            auto one = [&](float x) {                                             // a single element
                if (x > m) raise(x);
                seen = fmaxf(seen, x);
                F32x2 ignored = t2;
                pair(x, -INFINITY, f2_make(-m, -m), s2, ignored);
                if constexpr (ENT) masked_pair(x, -INFINITY, f2_make(-m, -m), t2);
            };
            // elements before the first whole vector
            if (part == 0 && tid < mine.head) one(Logit<T>::to_float(mine.x[tid]));
            bar.empty_sync(turn);                                                 // the finishing warp is done with this place
            int32_t left = (int32_t)(mine.v1 - mine.v0);                          // vectors of the share from this batch on
            uint32_t event = 2;                                                   // batches until the next event of the bound
            uint32_t v = mine.v0 + tid, batch = 0;                                // this thread's first vector of the batch
            const uint32_t raise_at = (2u << warp) + 1u;                          // the warp's turn to renew the bound
            float bound = NAN;                                                    // (none yet: nothing is noted)
            auto note = [&](uint32_t w, float top) {
                const uint32_t pos = atomicAdd(&r.count, 1u), bits = lp_note_bits<T>(p.V);
                if (pos < LP_NOTES) r.note[pos] = key_from_bits32(float_bits_exact(top)) >> bits << bits | w;
            };
            do {                                                                  // (an empty share still takes its batch)
                load_batch();
                lp_cp_wait<LP_STAGES - 1>();
                const uint4* in = ring + stage * LP_STEP + tid;
                // (vectors behind the share count as masked where maxima are taken, and are left out of the sums)
                const bool full = left >= (int32_t)LP_STEP;
                uint4 vec[U];
#pragma unroll
                for (int u = 0; u < U; ++u) vec[u] = in[u * LP_STREAM];
                if (!full) {
                    asm volatile("" ::: "memory");                                // (a branch, not sixteen selections per batch)
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (u * LP_STREAM + (int)tid >= left) vec[u] = Logit<T>::masked();
                }
                // One look at the batch's largest element decides whether the exponents' reference moves and whether any
                // vector has to be noted; both are rare, and decided by warp, which then stays together.
                typename Logit<T>::Top tops[U];
#pragma unroll
                for (int u = 0; u < U; ++u) tops[u] = Logit<T>::top_of(vec[u]);
                const float top = Logit<T>::value(Logit<T>::join(Logit<T>::join(tops[0], tops[1]), Logit<T>::join(tops[2], tops[3])));
                if (__any_sync(FULL_MASK, top > m))
                    raise(__uint_as_float(bits32_from_key(__reduce_max_sync(FULL_MASK, key_from_bits32(float_bits_exact(fmaxf(m, top)))))));
                if constexpr (TOPK) {
                    seen = fmaxf(seen, top);
                    if (__any_sync(FULL_MASK, top >= bound)) {
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (Logit<T>::value(tops[u]) >= bound) note(v + u * LP_STREAM, Logit<T>::value(tops[u]));
                        __syncwarp();
                    }
                }
                // (the batch's sums by themselves, then one addition: fewer terms meet a sum that is large already)
                const F32x2 minus_m = f2_make(-m, -m);
                F32x2 sb = f2_make(0.f, 0.f), tb = sb;
                if (full) {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        float x[VEC];
                        Logit<T>::unpack(vec[u], x);
#pragma unroll
                        for (int j = 0; j < VEC; j += 2) pair(x[j], x[j + 1], minus_m, sb, tb);
                    }
                } else {
#pragma unroll 1
                    for (int u = 0; u < U; ++u) {
                        if (u * LP_STREAM + (int)tid >= left) break;
                        float x[VEC];
                        Logit<T>::unpack(in[u * LP_STREAM], x);
#pragma unroll
                        for (int j = 0; j < VEC; j += 2) pair(x[j], x[j + 1], minus_m, sb, tb);
                    }
                    __syncwarp();
                }
                s2 = f2_add(s2, sb);
                if constexpr (ENT) {
                    // Masked elements in the batch (or NaN): t once more, slowly.
                    float a, b;
                    f2_split(tb, a, b);
                    if (__any_sync(FULL_MASK, isnan(a + b))) {
                        tb = f2_make(0.f, 0.f);
#pragma unroll 1
                        for (int u = 0; u < U; ++u) {
                            if (u * LP_STREAM + (int)tid >= left) break;
                            float x[VEC];
                            Logit<T>::unpack(in[u * LP_STREAM], x);
#pragma unroll
                            for (int j = 0; j < VEC; j += 2) masked_pair(x[j], x[j + 1], minus_m, tb);
                        }
                        __syncwarp();
                    }
                    t2 = f2_add(t2, tb);
                }
                if constexpr (TOPK) {
                    volatile float* bound_at = &r.bound;
                    if (batch == 0) {
                        lp_write_slot(seen, tid, slot_lanes, sh);                 // (all slots of the row before anyone reads one)
                        if (parts == 1) {
                            bound = lp_first_bound(seen, p.k, sh, bar);
                        } else {
                            // k of the row's elements reach the least of the parts' (k / parts)-th largest, a much better
                            // bound than a part's own k-th unless some part is masked: then the best of those instead.
                            bound = lp_exchange(lp_first_bound(seen, (p.k + parts - 1) >> p.parts_log2, sh, bar), false);
                            if (bound == LOWEST) bound = lp_exchange(lp_first_bound(seen, p.k, sh, bar), true);
                        }
                        if (tid == 0) *bound_at = bound;                          // (nobody else writes it before two more batches)
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (Logit<T>::value(tops[u]) >= bound) note(v + u * LP_STREAM, Logit<T>::value(tops[u]));
                        __syncwarp();
                    }
                    // After 2, 4, 8, ... batches the slots are written again, and a batch later one warp renews the bound.
                    if (++batch == event) {
                        if (batch & 1) {
                            if (batch == raise_at) {
                                const float higher = lp_slot_bound(*bound_at, p.k, slot_lanes, sh);
                                if (lane == 0 && higher > *bound_at) *bound_at = higher;
                            }
                            event = 2 * (batch - 1);
                        } else {
                            lp_write_slot(seen, tid, slot_lanes, sh);
                            event = batch + 1;
                        }
                    }
                    if (batch > 2) bound = *bound_at;
                }
                stage = stage + 1 == LP_STAGES ? 0 : stage + 1;
                v += LP_STEP;
                left -= (int32_t)LP_STEP;
            } while (left > 0);
            mine.set(p, row, part);                                        // (computed again rather than kept)
            // elements behind the last whole vector
            const uint32_t tail = mine.head + mine.nvec * VEC;
            if (part == parts - 1 && tail + tid < p.V) one(Logit<T>::to_float(mine.x[tail + tid]));

            // join the lanes' parts, in a fixed order
            LpStats st;
            st.m = m;
            float a, b;
            f2_split(s2, a, b);
            st.s = a + b;
            f2_split(t2, a, b);
            st.t = a + b;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                LpStats o;
                o.m = __shfl_xor_sync(FULL_MASK, st.m, d);
                o.s = __shfl_xor_sync(FULL_MASK, st.s, d);
                o.t = ENT ? __shfl_xor_sync(FULL_MASK, st.t, d) : 0.f;
                st = (lane & d) ? lp_join(o, st, c) : lp_join(st, o, c);
            }
            if (lane == 0) r.stats[warp] = st;
            bar.full_arrive(turn);
            if (parts > 1) cluster.sync();
            turn ^= 1;
        }
        lp_cp_wait<0>();
    }
    if (parts > 1) cluster.sync();                                                // no CTA leaves while its memory is written
}

// ---------------------------------------------------------------------------------------------------------------------
// Gradient.  With upstream gradients g_lp (of the token's log probability), g_H, g_lse and g_j (of the alternatives'),
//   dL/dx_v = (1/T) [ -p_v (G + g_H (ln p_v + H)) + g_lp 1[v = token] + sum_j g_j 1[v = i_j] ],   G = g_lp + sum_j g_j - g_lse,
// p_v = e^(x_v / T - lse): one read and one write of the matrix; the picked entries are written again behind a barrier.
// Bound by HBM: 4096 x 131072 bf16 (2.1 GB) in 344 to 358 us, 6.0 to 6.2 TB/s, 0.92 to 0.95 of a copy's rate; 256 threads with 64 bytes each in flight, a
// grid over chunks of rows.
struct LpGradParams {
    const void* logits;
    void* grad;
    int64_t rows, row_stride, grad_stride;
    uint32_t V, k, chunks;               // chunks per row
    uint32_t chunk;                      // elements per chunk
    float scale, unscale;                // 1 / T, and its reciprocal
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

// ln p = (x - from) / T - lse - rest, and of that -rest log2(e); (G + g_H (H - rest)) / T; g_H / T
struct LgRow { float from, lse, rest2, whole, g_h; };

__device__ __forceinline__ float lg_dense(float x, const LgRow& r, float scale) {
    const float a = fmaf(x - r.from, scale, -r.lse);
    const float q = exp2_approx(fmaf(a, LOG2E, r.rest2));
    return -q * fmaf(r.g_h, fmaxf(a, FAR_BELOW), r.whole);
}

// SHIFTED: the logits' rows start at other offsets within 16 bytes than the gradient's (a build of its own: its registers
// would cost the other one an eighth of its threads, 2048 x 131072 bf16 175 us instead of 164; four CTAs of it to an SM, 1024 x
// 131072 bf16 100 us, three 112).
template <typename T, bool SHIFTED>
__global__ void __launch_bounds__(LG_THREADS, SHIFTED ? 4 : 5) logprobs_grad_kernel(const LpGradParams p) {
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
    const bool given = p.g_logprob && token >= 0 && token < (int64_t)p.V;      // there is something to add to the token's entry
    const float g_lp = given ? p.g_logprob[row] : 0.f;
    const float scale = p.scale;
    float g_sum = 0.f;
    if (p.g_top) {
        float g = 0.f;
        for (uint32_t j = tid; j < p.k; j += LG_THREADS) {
            const int64_t i = p.top_tokens[row * p.k + j];
            if (i >= 0 && i < (int64_t)p.V) g += p.g_top[row * p.k + j];           // (a place without a token has no gradient)
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) g += __shfl_xor_sync(FULL_MASK, g, d);
        if ((tid & 31) == 0) s_sum[tid >> 5] = g;
        __syncthreads();
        for (int w = 0; w < LG_THREADS / 32; ++w) g_sum += s_sum[w];
    }
    LgRow r;
    r.lse = p.lse[row];
    float rest = p.lse_rest ? p.lse_rest[row] : 0.f;
    const float g_h = p.g_entropy ? p.g_entropy[row] : 0.f;
    const float whole = g_lp + g_sum - (p.g_lse ? p.g_lse[row] : 0.f);
    const bool empty = isinf(r.lse);                       // nothing but -inf in the row, or more than fp32 holds: no gradient
    const bool huge = p.lse_rest && fabsf(r.lse) >= LP_HUGE;                      // see lp_rest
    r.from = huge && !empty ? lp_max_of(r.lse, rest, p.unscale) : 0.f;
    r.lse = empty ? INFINITY : huge ? rest : r.lse;        // (empty: a is -inf for every element, its exponential and the factors 0)
    rest = huge ? 0.f : rest;
    r.rest2 = -rest * LOG2E;
    r.whole = empty ? 0.f : (whole + (p.g_entropy ? g_h * (p.entropy[row] - rest) : 0.f)) * scale;
    r.g_h = empty ? 0.f : g_h * scale;

    const uint32_t e0 = chunk * p.chunk, e1 = min(p.V, e0 + p.chunk);
    // Vectors are those of the gradient's rows; where the logits' rows start at another offset, each is put together from two
    // of theirs (2048 x 131072 bf16, logits one element off: 190 us, and 771 element by element).
    const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(y + e0) & 15u);
    auto scalar = [&](uint32_t i) { y[i] = Logit<T>::from_float(lg_dense(Logit<T>::to_float(x[i]), r, scale)); };
    const uint32_t head = min(e1, e0 + (mis ? (16u - mis) / (uint32_t)sizeof(T) : 0u));
    const uint32_t nvec = (e1 - head) / VEC, tail = head + nvec * VEC;
    if (e0 + tid < head) scalar(e0 + tid);
    if (tail + tid < e1) scalar(tail + tid);
    auto put = [&](uint32_t v, const uint4& in) {
        float f[VEC];
        Logit<T>::unpack(in, f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = lg_dense(f[j], r, scale);
        st_stream_u4(y + head + (size_t)v * VEC, Logit<T>::pack(f));
    };
    if constexpr (!SHIFTED) {
        // (the gradient may take the logits' place, so that these are not read through the read-only path)
        for (uint32_t v = tid; v < nvec; v += LG_THREADS * U) {
            uint4 in[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * LG_THREADS < nvec) in[u] = ld_once_u4(x + head + (size_t)(v + u * LG_THREADS) * VEC);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * LG_THREADS < nvec) put(v + u * LG_THREADS, in[u]);
        }
    } else {
        // (the 16 bytes in which an element of the row lies can be read whole)
        const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(x + head) & ~(uintptr_t)15u);
        const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(x + head) & 15u);
        const uint32_t words = shift >> 2, bits = (shift & 3u) * 8u, more = shift ? 1u : 0u;
        for (uint32_t v = tid; v < nvec; v += LG_THREADS * U) {
            uint4 lo[U], hi[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * LG_THREADS < nvec) {
                    lo[u] = __ldg(from + v + u * LG_THREADS);
                    hi[u] = __ldg(from + v + u * LG_THREADS + more);
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * LG_THREADS < nvec) {
                    const uint32_t w[8] = {lo[u].x, lo[u].y, lo[u].z, lo[u].w, hi[u].x, hi[u].y, hi[u].z, hi[u].w};
                    uint32_t a[6], b[5];
#pragma unroll
                    for (int j = 0; j < 6; ++j) a[j] = words & 2u ? w[j + 2] : w[j];
#pragma unroll
                    for (int j = 0; j < 5; ++j) b[j] = words & 1u ? a[j + 1] : a[j];
                    put(v + u * LG_THREADS, make_uint4(__funnelshift_r(b[0], b[1], bits), __funnelshift_r(b[1], b[2], bits),
                                                       __funnelshift_r(b[2], b[3], bits), __funnelshift_r(b[3], b[4], bits)));
                }
        }
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
