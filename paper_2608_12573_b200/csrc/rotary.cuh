// Rotary positions.  Of every head, pair i of the first 2 * pairs elements is turned by the angle a = position * frequency_i:
//   y_1 = m (x_1 cos a - x_2 sin a),   y_2 = m (x_2 cos a + x_1 sin a);   the rest of the head is copied bit for bit.
// The transpose of a turn is the turn by -a, so the gradient is the same kernel with `inverse` set.
//
// Angles.  At position 10^6 an fp32 product is off by 0.06 radians.  A frequency is therefore held as a 64-bit fraction of a
// full turn, and position * fraction is one 64-bit integer product whose wrap-around is the reduction, with no 64-bit floating-point
// arithmetic per angle but the conversion.  An angle is off by 2^-52 of itself (the frequency in turns: a rounded product with a rounded
// constant, 1.55 * 2^-53), by |position| * 2^-61 radians (the fraction's last bit) and by 2^-30 (32 bits of the phase are kept).
//
// Both operators are bound by HBM: each element is read and written once.  The angles of a token serve all its heads, so a
// CTA finds those of its tokens once, into shared memory, and a thread keeps the few that its vectors need in registers over
// four heads, whose loads are in flight together.  CTAs to an SM: three where a chunk is two vectors, four where it is one
// (16384 x 32 x 128 bf16 turned by halves, forward and backward: 104 us with three, 128 with four, whose registers spill; 16384
// ragged rows of 80 interleaved f16 heads appended: 129 and 122).  Angles found by each thread for itself, without barriers,
// over more heads: 103 and 155.
#pragma once

#include "logits.cuh"

namespace profk {

constexpr int RO_THREADS = 256;
constexpr int RO_TOKENS = 32;             // tokens of a CTA at most
constexpr int RO_MAX_PAIRS = 512;
constexpr int RO_ANGLES = 4096;           // of a CTA at most: 32 KB

template <typename T>
struct RoRows {                           // rows (outer, inner, head) of `dim` elements, strides in elements
    T* p;
    int64_t outer, inner, head;
    __device__ __forceinline__ T* at(int64_t o, int64_t i, int64_t h) const { return p + o * outer + i * inner + h * head; }
};

template <typename T>
struct RoParams {
    RoRows<const T> q;                    // what is turned and given back
    T* out;                               // rows x heads x dim, dense
    int64_t rows, inner;                  // rows = outer * inner
    int32_t heads, dim, pairs, tokens_per_cta;
    const double* frequencies;
    float magnitude;                      // of the turn; negative sine: see `inverse`
    bool inverse;
    const int64_t* positions;             // null: the places in the cache
    int64_t pos_outer, pos_inner;
    // what goes into the pages (kv_heads = 0: nothing)
    RoRows<const T> k, v;
    int32_t kv_heads, seqs, page_size, pages, width;
    T* k_pages;
    T* v_pages;
    int64_t kp_page, kp_head, kp_token, vp_page, vp_head, vp_token;
    const int32_t* tables;
    int64_t table_stride;
    const int32_t* lengths;               // null: positions only
    const int32_t* starts;                // null: sequence s has the rows [s * inner, (s + 1) * inner)
};

struct RoToken {
    int64_t outer, inner, position;
    int64_t k_at, v_at;                   // offset of the token's row of head 0 in the pages; -1: it has no place
    int32_t held;                         // whether a sequence holds this row
};

// How many entries of `starts` (ascending, n of them) are <= row, found by a warp, 32 probes at a time.
__device__ __forceinline__ int32_t starts_up_to(const int32_t* starts, int32_t n, int64_t row) {
    int32_t lo = 0, hi = n;
    const int32_t lane = (int32_t)lane_id();
    while (hi - lo > 32) {
        const int32_t step = (hi - lo + 31) / 32;
        const int64_t at = (int64_t)lo + (int64_t)lane * step;
        const int32_t c = __popc(__ballot_sync(FULL_MASK, at < hi && starts[at] <= row));
        if (c == 0) return lo;
        lo += (c - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo + __popc(__ballot_sync(FULL_MASK, lo + lane < hi && starts[lo + lane] <= row));
}

// (cos, sin) of position * frequency radians, times the magnitude.
__device__ __forceinline__ float2 ro_turn(int64_t position, double frequency, float magnitude, bool inverse) {
    double turns = frequency * 0.15915494309189535;                      // 1 / (2 pi)
    turns -= rint(turns);
    const int64_t fraction = __double2ll_rn(turns * 18446744073709551616.0);
    const uint64_t phase = (uint64_t)position * (uint64_t)fraction;
    const uint32_t top = (uint32_t)((phase + 0x80000000ull) >> 32);       // 2^-32 turns
    const uint32_t quarter = (top + 0x20000000u) >> 30;                   // the nearest quarter turn, and what is left of it
    const float rest = (float)(int32_t)(top - (quarter << 30)) * 4.656612873077393e-10f;      // in half turns: |rest| <= 1/4
    float s, c;
    sincospif(rest, &s, &c);
    if (quarter & 1u) { const float t = c; c = -s; s = t; }
    if (quarter & 2u) { c = -c; s = -s; }
    return make_float2(c * magnitude, (inverse ? -s : s) * magnitude);
}

// (Rounded the same way in every build, so that results do not depend on alignment.)
__device__ __forceinline__ void ro_apply(const float2& turn, float& first, float& second) {
    const float x = first, y = second;
    first = __fmaf_rn(x, turn.x, -__fmul_rn(y, turn.y));
    second = __fmaf_rn(y, turn.x, __fmul_rn(x, turn.y));
}

// VEC elements at a time: a 16-byte vector, or a single element where alignment or sizes allow no more.
template <typename T, int VEC> struct RoVec;
template <typename T> struct RoVec<T, 1> {
    T raw;
    __device__ __forceinline__ void load(const T* p) { raw = *p; }
    __device__ __forceinline__ void store(T* p) const { *p = raw; }
    __device__ __forceinline__ void unpack(float (&x)[1]) const { x[0] = Logit<T>::to_float(raw); }
    __device__ __forceinline__ void pack(const float (&x)[1]) { raw = Logit<T>::from_float(x[0]); }
};
template <typename T, int VEC> struct RoVec {
    static_assert(VEC == Logit<T>::VEC, "a vector is 16 bytes");
    uint4 raw;
    __device__ __forceinline__ void load(const T* p) { raw = ld_stream_u4(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = raw; }
    __device__ __forceinline__ void unpack(float (&x)[VEC]) const { Logit<T>::unpack(raw, x); }
    __device__ __forceinline__ void pack(const float (&x)[VEC]) { raw = Logit<T>::pack(x); }
};

// The vectors a thread handles of each head: number c of them.  Half layout: a pair of vectors (or one that is copied);
// interleaved: one vector (of single elements: a pair, or one that is copied).
template <typename T, int VEC, bool INTER>
struct RoChunk {
    static constexpr int PER = INTER && VEC > 1 ? VEC / 2 : VEC;         // pairs of a turned chunk
    static constexpr bool TWO = !INTER || VEC == 1;                      // a turned chunk is two vectors
    int32_t first, second, pair;          // offsets in the head; first pair
    bool turned;
    __device__ __forceinline__ RoChunk(int32_t c, int32_t pairs) {
        const int32_t count = pairs / PER;                               // turned chunks
        turned = c < count;
        pair = c * PER;
        if (!turned) first = 2 * pairs + (c - count) * VEC;
        else if (INTER) first = 2 * pair;
        else first = pair;
        second = INTER ? first + 1 : first + pairs;
    }
};
template <int VEC, bool INTER>
__host__ __device__ __forceinline__ int32_t ro_chunks(int32_t dim, int32_t pairs) {
    return pairs / (INTER && VEC > 1 ? VEC / 2 : VEC) + (dim - 2 * pairs) / VEC;
}

// HB heads of a token are one thread's unit: their loads are in flight together.  (Few tokens: HB = 1, more threads.)
template <typename T, int VEC, bool INTER, int HB>
__global__ void __launch_bounds__(RO_THREADS, INTER ? 4 : 3) rotary_kernel(const RoParams<T> p) {
    using Chunk = RoChunk<T, VEC, INTER>;
    extern __shared__ float2 angles[];                                   // tokens_per_cta x pairs
    __shared__ RoToken tokens[RO_TOKENS];
    pdl_wait();
    pdl_launch_dependents();
    const int64_t row0 = (int64_t)blockIdx.x * p.tokens_per_cta;
    const int32_t n = (int32_t)min((int64_t)p.tokens_per_cta, p.rows - row0);
    for (int32_t i = (int32_t)threadIdx.x / 32; i < n; i += RO_THREADS / 32) {    // a warp to a token
        const int64_t row = row0 + i;
        RoToken t;
        t.outer = row / p.inner;
        t.inner = row - t.outer * p.inner;
        t.k_at = t.v_at = -1;
        t.held = 1;
        int64_t place = 0;
        int32_t seq = (int32_t)t.outer;
        if (p.lengths) {
            if (p.starts) {
                seq = starts_up_to(p.starts, p.seqs + 1, row) - 1;
                t.held = seq >= 0 && seq < p.seqs;
                if (t.held) place = (int64_t)p.lengths[seq] - ((int64_t)p.starts[seq + 1] - row);
            } else {
                place = (int64_t)p.lengths[seq] - p.inner + t.inner;
            }
            if (t.held && place >= 0 && place < (int64_t)p.width * p.page_size) {
                const int32_t at = (int32_t)place;
                const int32_t page = p.tables[seq * p.table_stride + at / p.page_size], slot = at % p.page_size;
                if (page >= 0 && page < p.pages) {
                    t.k_at = page * p.kp_page + slot * p.kp_token;
                    t.v_at = page * p.vp_page + slot * p.vp_token;
                }
            }
        }
        t.position = p.positions ? p.positions[t.outer * p.pos_outer + t.inner * p.pos_inner] : place;
        if (lane_id() == 0) tokens[i] = t;
    }
    __syncthreads();
    for (int32_t i = (int32_t)threadIdx.x; i < n * p.pairs; i += RO_THREADS) {
        const int32_t t = i / p.pairs;
        angles[i] = ro_turn(tokens[t].position, p.frequencies[i - t * p.pairs], p.magnitude, p.inverse);
    }
    __syncthreads();
    const int32_t chunks = ro_chunks<VEC, INTER>(p.dim, p.pairs), heads = p.heads + 2 * p.kv_heads;
    const int32_t units = (heads + HB - 1) / HB, items = n * units * chunks;
    for (int32_t item = (int32_t)threadIdx.x; item < items; item += RO_THREADS) {
        const int32_t unit = item / chunks, c = item - unit * chunks, token = unit / units, h0 = (unit - token * units) * HB;
        const Chunk chunk(c, p.pairs);
        const RoToken& t = tokens[token];
        RoVec<T, VEC> a[HB], b[HB];
        T* to[HB];
        bool turn[HB];
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int32_t h = h0 + i;
            const T* from = nullptr;
            to[i] = nullptr;
            turn[i] = chunk.turned;
            if (h < p.heads) {
                from = p.q.at(t.outer, t.inner, h);
                to[i] = p.out + ((row0 + token) * p.heads + h) * p.dim;
            } else if (h < p.heads + p.kv_heads) {
                from = p.k.at(t.outer, t.inner, h - p.heads);
                if (t.k_at >= 0) to[i] = p.k_pages + t.k_at + (h - p.heads) * p.kp_head;
            } else if (h < heads) {
                from = p.v.at(t.outer, t.inner, h - p.heads - p.kv_heads);
                turn[i] = false;
                if (t.v_at >= 0) to[i] = p.v_pages + t.v_at + (h - p.heads - p.kv_heads) * p.vp_head;
            }
            if (to[i]) {
                a[i].load(from + chunk.first);
                if (Chunk::TWO && chunk.turned) b[i].load(from + chunk.second);
            }
        }
        float2 w[Chunk::PER];
        if (chunk.turned) {
#pragma unroll
            for (int j = 0; j < Chunk::PER; ++j) w[j] = angles[token * p.pairs + chunk.pair + j];
        }
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            if (!to[i]) continue;
            if (!t.held) {                                               // a row that no sequence holds comes back as zeros
                float zero[VEC] = {};
                a[i].pack(zero);
                b[i] = a[i];
            } else if (turn[i]) {
                float x[VEC];
                a[i].unpack(x);
                if constexpr (Chunk::TWO) {
                    float y[VEC];
                    b[i].unpack(y);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) ro_apply(w[j], x[j], y[j]);
                    b[i].pack(y);
                } else {
#pragma unroll
                    for (int j = 0; j < Chunk::PER; ++j) ro_apply(w[j], x[2 * j], x[2 * j + 1]);
                }
                a[i].pack(x);
            }
            a[i].store(to[i] + chunk.first);
            if (Chunk::TWO && chunk.turned) b[i].store(to[i] + chunk.second);
        }
    }
}

}  // namespace profk
