// Attention of one new token per sequence over a paged key-value cache:
//   out_h = sum_j p_j v_j,   p = softmax_j(scale q_h . k_j),   lse_h = ln sum_j e^(scale q_h . k_j),   j < length.
//
// The cache is read once and every key meets the few query heads that share it, so the kernel is bound by HBM (4 dim
// bytes and 4 dim G operations per token and key-value head).  The work is the list of (sequence, key-value head, tile of
// 16 tokens), cut into one contiguous share per warp whatever the lengths.  A warp that holds only part of a (sequence,
// head) leaves its running maximum, sum and unnormalised output in scratch memory; at its end a CTA joins the parts of its
// own warps, and a second, small kernel those of several CTAs, always in order.  A barrier every few tiles keeps the warps
// of an SM together: left to themselves some finished their equal shares in two thirds of the others' time (200 sequences of
// 17 to 700 tokens: 42 us against 75), and the SM was half idle in the end.
//
// A warp works by itself: its tiles come through a ring of its own in shared memory (cp.async, no barrier), and it
// multiplies with the warp-level matrix instruction, tokens (and then dimensions) along its 16 rows and query heads along
// its 8 columns: K Q^T, then V^T P^T.  More than 16 heads to a key take a pass over the key-value head for each 16, as tiles
// of their own in other warps' shares, so that the cache is read again from L2 or HBM and the arithmetic, not HBM, is the bound
// (16 sequences of 16384 tokens, one key-value head: 16 heads 50 us, 32 67, 64 108).  The few heads that share a key are the narrow side of the product, far below the 128
// rows that a tcgen05 tile wants, and the tensor pipe is not what bounds it.
#pragma once

#include "logits.cuh"

namespace profk {

constexpr int PA_SUB = 16;                              // tokens per step of the matrix instruction
constexpr int PA_ROWS = 16;                             // most query heads per pass over a key-value head
constexpr int PA_PACE = 4;                              // tiles between two barriers of a CTA, which keep its reads close together
                                                        // (4 x 131072 tokens: 287 us; every 8, 16, 64 tiles: 292, 295, 301;
                                                        // 290 since a tile's products are summed apart)

template <int D> struct PaShape {
    // One CTA per SM, 192 KB of rings.  A tile is 8 KB of keys and values or more: with 16 tokens of 64 dimensions at a time
    // the arithmetic around them held the stream to 5.5 TB/s.
    static constexpr int SUBS = D == 64 ? 2 : 1;        // steps per tile
    static constexpr int TILE = PA_SUB * SUBS;          // tokens per tile
    static constexpr int WARPS = D == 256 ? 4 : 8;
    static constexpr int THREADS = WARPS * 32;
    static constexpr int STAGES = 3;                    // of a warp's ring
    static constexpr int SUB_BYTES = PA_SUB * D * 2 * 2;                                 // keys, then values
    static constexpr int STAGE_BYTES = SUB_BYTES * SUBS;
    static constexpr size_t SMEM = (size_t)WARPS * STAGES * STAGE_BYTES;
    static constexpr int SLOT = PA_ROWS * (D + 2);      // floats of a part: output, maxima, sums
    static constexpr int SLOTS = 2 * WARPS + 2;         // of a CTA: for each warp, then for the CTA, its first and its last stream
};

struct PaMeta { int32_t seq, head, heads, last; };      // the parts of `heads` heads of seq: this CTA's to CTA `last`'s; seq < 0: none

struct PaParams {
    const void* q;
    const void* k;
    const void* v;
    int64_t q_seq, q_head;                              // strides in elements
    int64_t k_page, k_head, k_token, v_page, v_head, v_token;
    const int32_t* tables;
    int64_t table_stride;
    const int32_t* lengths;
    int32_t seqs, heads, kv_heads, group, dim, page_size, pages, width;
    int32_t blocks, rows;                               // passes per key-value head, query heads per pass (<= PA_ROWS)
    int32_t page_shift;                                 // log2 of the page size, or -1
    // The page size is a multiple of 16: a step's tokens lie in one page, whose number is looked up once instead of per token
    // (32 ragged sequences, 16 heads to a key: 119 us against 127, 8 heads: 101 against 103).
    int32_t one_page;
    float scale;
    void* out;                                          // seqs x heads x dim
    float* lse;                                         // seqs x heads
    float* parts;                                       // SLOTS slots per CTA
    PaMeta* meta;                                       // one per CTA
};

// Weights are e^(score - reference) 2^SHIFT, and the reference may lag the largest score so far by up to 2^LAG.  fp16 ends at
// 2^-24: the pair of numbers that a weight is split into for the second product is off by up to 2^-25 of it, so that the
// weights are lifted as far as 65504 allows, and each is off by 2^-39 of the largest at most, or by 2^-22 of itself (unlifted
// and with a lag of 2^8, tokens 2^-24.4 below a sink counted a third too much and those from 2^-25 on not at all).  bf16 has
// fp32's range.
template <typename T> struct PaWeights { static constexpr float LAG = 8.f, SHIFT = 0.f, UNIT = 1.f; };
template <> struct PaWeights<__half> { static constexpr float LAG = 1.f, SHIFT = 14.f, UNIT = 16384.f; };      // UNIT = 2^SHIFT
// lse of a reference and a sum of weights.
template <typename T>
__device__ __forceinline__ float pa_lse(float m, float sum, float scale) {
    return sum == 0.f ? -INFINITY : fmaf(m, scale, logf(sum * (1.f / PaWeights<T>::UNIT)));
}

template <typename T>
__device__ __forceinline__ void pa_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void pa_mma<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void pa_mma<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two floats to a pair of T (the first in the low half), and what that rounding left off as another pair.
template <typename T>
__device__ __forceinline__ uint32_t pa_pack(float a, float b);
template <>
__device__ __forceinline__ uint32_t pa_pack<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pa_pack<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T>
__device__ __forceinline__ float2 pa_unpack(uint32_t w);
template <>
__device__ __forceinline__ float2 pa_unpack<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <>
__device__ __forceinline__ float2 pa_unpack<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

__device__ __forceinline__ void pa_ldmatrix(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void pa_ldmatrix_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// 16 bytes to shared memory, or 16 zero bytes (nothing is read then).
__device__ __forceinline__ void pa_cp_async(uint32_t smem, const void* gmem, bool read) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(gmem), "r"(read ? 16 : 0) : "memory");
}
__device__ __forceinline__ void pa_cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void pa_cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ int32_t pa_length(const PaParams& p, int32_t seq) {
    const int64_t room = (int64_t)p.width * p.page_size;
    return (int32_t)max((int64_t)0, min((int64_t)p.lengths[seq], room));
}

// A place in the list of tiles: sequence by sequence, head by head (and pass by pass), tile by tile.
template <int TILE>
struct PaCursor {
    int32_t seq, head, block, tile, tiles, len;
    // To the next tile, past empty sequences.
    __device__ __forceinline__ void next(const PaParams& p) {
        if (++tile < tiles) return;
        tile = 0;
        if (++block < p.blocks) return;
        block = 0;
        if (++head < p.kv_heads) return;
        head = 0;
        do {
            if (++seq >= p.seqs) { tiles = 0; return; }
            len = pa_length(p, seq);
            tiles = (len + TILE - 1) / TILE;
        } while (tiles == 0);
    }
    __device__ __forceinline__ int32_t first_head(const PaParams& p) const { return head * p.group + block * p.rows; }
    __device__ __forceinline__ int32_t heads(const PaParams& p) const { return min(p.rows, p.group - block * p.rows); }
};

// What the parts of a warp's share are, for the join at the CTA's end.
struct PaShare {
    int32_t first;                                      // its first stream began in an earlier share: heads of that stream, else 0
    int32_t first_ends;                                 // ... and ended in this one
    int32_t seq, head, heads;                           // the stream that began here and goes on behind it; heads 0: none
    int32_t last;                                       // the share that stream ends in
};

// Parts of consecutive warps that belong to one stream; `before`: heads of the chains before it.
struct PaChain { int32_t from, last, heads, before; bool inside, final; };

// Transposes an 8 x 8 matrix of 16-bit numbers held by the warp (lane 4 r + q: row r, columns 2 q and 2 q + 1).
__device__ __forceinline__ uint32_t pa_transpose(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// A list of `total` tiles in `shares` shares of equal length, the first `more` of them one tile longer.
struct PaShares {
    long long each;
    int32_t more, n;
    __device__ __forceinline__ PaShares(long long total, int32_t warps) {
        n = (int32_t)max(1LL, min((long long)warps, total));
        each = total < 0x7FFFFFFF ? (long long)((uint32_t)total / (uint32_t)n) : total / n;
        more = (int32_t)(total - each * n);
    }
    __device__ __forceinline__ long long begin(int32_t i) const { return i < n ? each * i + min(i, more) : each * n + more; }
    __device__ __forceinline__ int32_t of(long long unit) const {             // the share that holds a tile
        const long long longer = (each + 1) * more;
        return (int32_t)(unit < longer ? unit / (each + 1) : more + (unit - longer) / each);
    }
};

// N8: groups of eight query heads per pass (rows <= 8 N8).  Up to 8 heads to a key take N8 = 1: 200 short sequences with
// one 77 us, with N8 = 2 92; 32 ragged ones with eight 101 and 106.
template <typename T, int D, int N8>
__global__ void __launch_bounds__(PaShape<D>::THREADS, 1) paged_attention_kernel(const PaParams p) {
    using Shape = PaShape<D>;
    constexpr int STAGES = Shape::STAGES, CH = D / 8, KSTEPS = D / 16, MT = D / 16, WARPS = Shape::WARPS, THREADS = Shape::THREADS,
                  SUBS = Shape::SUBS, TILE = Shape::TILE, AT_ONCE = D > 64 && N8 == 2 ? 2 : 4;
    constexpr int ROWS_PER_LOAD = 32 / CH;                                   // token rows that one warp-wide copy covers
    constexpr int LOADS = PA_SUB / ROWS_PER_LOAD;
    extern __shared__ __align__(512) unsigned char pa_dyn[];           // (512: the longest row; see the exclusive ors below)
    __shared__ uint32_t s_mask[WARPS][STAGES][SUBS];
    __shared__ long long s_scan[WARPS], s_start[WARPS];
    __shared__ int32_t s_seq[WARPS];
    __shared__ PaShare s_share[WARPS];
    __shared__ PaChain s_chain[WARPS + 1];
    __shared__ float s_max[WARPS][2][PA_ROWS], s_sum[WARPS][2][PA_ROWS];      // of the warps' parts

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, quad = lane & 3;
    const int32_t streams = p.kv_heads * p.blocks;
    const float c = p.scale * LOG2E;
    // Lengths and page tables on their way into L2 while the kernel before this one ends (a prefetch reads nothing).
    {
        const int64_t lines = ((int64_t)p.seqs * 4 + 127) / 128, row_lines = ((int64_t)p.width * 4 + 127) / 128;
        for (int64_t i = (int64_t)blockIdx.x * THREADS + tid; i < lines + p.seqs * row_lines && i < (1 << 20); i += (int64_t)gridDim.x * THREADS) {
            const char* at = i < lines ? reinterpret_cast<const char*>(p.lengths) + i * 128
                                       : reinterpret_cast<const char*>(p.tables + (i - lines) / row_lines * p.table_stride) + (i - lines) % row_lines * 128;
            asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
        }
    }
    pdl_wait();
    pdl_launch_dependents();

    // where the sequences' tiles begin in the list: each thread sums a run of sequences
    const int32_t per = (p.seqs + THREADS - 1) / THREADS;
    const int32_t run0 = min(p.seqs, tid * per), run1 = min(p.seqs, run0 + per);
    auto tiles_of = [&](int32_t s) { return (long long)((pa_length(p, s) + TILE - 1) / TILE) * streams; };
    long long mine = 0;
    for (int32_t s = run0; s < run1; ++s) mine += tiles_of(s);
    long long incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long n = __shfl_up_sync(FULL_MASK, incl, d);
        if (lane >= d) incl += n;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) incl += s_scan[w];
        total += s_scan[w];
    }
    const PaShares shares(total, gridDim.x * WARPS);
    const int32_t me = blockIdx.x * WARPS + warp;
    // who begins where: the threads whose run of sequences holds the first tile of one of the CTA's shares say so
    const long long cta0 = shares.begin(blockIdx.x * WARPS), cta1 = shares.begin((blockIdx.x + 1) * WARPS);
    if (incl - mine < cta1 && incl > cta0) {
        for (int w = 0; w < WARPS; ++w) {
            const long long u = shares.begin(blockIdx.x * WARPS + w);
            if (u < incl - mine || u >= incl) continue;
            long long at = incl - mine;
            int32_t s = run0;
            for (;; ++s) {
                const long long n = per > 1 ? tiles_of(s) : mine;
                if (u < at + n) break;
                at += n;
            }
            s_seq[w] = s;
            s_start[w] = at;
        }
    }
    __syncthreads();
    const long long u0 = shares.begin(me), u1 = shares.begin(me + 1);
    // barriers of the CTA, the same number for all of its warps
    const int32_t turns = (int32_t)((shares.begin(blockIdx.x * WARPS + 1) - cta0) / PA_PACE);
    int32_t turn = 0;
    PaShare share{0, 0, 0, 0, 0, 0};
    float* const slots = p.parts + (int64_t)blockIdx.x * Shape::SLOTS * Shape::SLOT;
    if (u0 < u1) {
    PaCursor<TILE> work;
    work.seq = s_seq[warp];
    work.len = pa_length(p, work.seq);
    work.tiles = (work.len + TILE - 1) / TILE;
    const uint32_t in_seq = (uint32_t)(u0 - s_start[warp]), stream0 = in_seq / (uint32_t)work.tiles;   // (a sequence's tiles: less than 2^32)
    work.tile = (int32_t)(in_seq - stream0 * (uint32_t)work.tiles);
    work.head = (int32_t)stream0 / p.blocks;
    work.block = (int32_t)stream0 - work.head * p.blocks;
    const uint32_t count = (uint32_t)(u1 - u0);

    // loading side
    PaCursor<TILE> load = work;
    uint32_t loaded = 0;
    int load_stage = 0;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(pa_dyn) + warp * STAGES * Shape::STAGE_BYTES;
    const int chunk = lane % CH, row0 = lane / CH;                            // (CH = 32: one row per copy)
    const bool chunk_in = chunk * 8 < p.dim;
    const uint32_t to0 = row0 * (D * 2) + ((chunk ^ (row0 & 7)) << 4);
    auto page_number = [&](int32_t t) { return p.page_shift >= 0 ? t >> p.page_shift : t / p.page_size; };
    // of the sequence and head that is being loaded: its row of the table, and the lane's place in page 0, token 0
    const int32_t* table = nullptr;
    const char* k_base = nullptr;
    const char* v_base = nullptr;
    auto new_stream = [&]() {
        table = p.tables + load.seq * p.table_stride;
        const int32_t in = chunk_in ? chunk * 8 : 0;
        k_base = reinterpret_cast<const char*>(reinterpret_cast<const T*>(p.k) + load.head * p.k_head + row0 * p.k_token + in);
        v_base = reinterpret_cast<const char*>(reinterpret_cast<const T*>(p.v) + load.head * p.v_head + row0 * p.v_token + in);
    };
    new_stream();
    const int64_t k_page = p.k_page * 2, v_page = p.v_page * 2;               // bytes
    const uint32_t k_token = (uint32_t)p.k_token * 2, v_token = (uint32_t)p.v_token * 2;    // (one_page: a page's tokens span less than 2^32 bytes)
    // page of the lane's token of a step (one_page: of the step's first token); -1: no token, or no page
    auto page_of = [&](const PaCursor<TILE>& at, int sub) -> int32_t {
        const int32_t t = at.tile * TILE + sub * PA_SUB + (p.one_page ? 0 : (lane & 15));
        if (t >= at.len) return -1;
        const int32_t page = table[page_number(t)];
        return page >= 0 && page < p.pages ? page : -1;
    };
    int32_t page[SUBS];
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) page[sub] = page_of(load, sub);
    auto load_tile = [&]() {
        if (loaded < count) {
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                const int32_t t0 = load.tile * TILE + sub * PA_SUB;
                const uint32_t base = ring + load_stage * Shape::STAGE_BYTES + sub * Shape::SUB_BYTES;
                if (p.one_page) {
                    const int32_t slot = t0 - page_number(t0) * p.page_size;
                    const int32_t n = page[sub] < 0 ? 0 : min(PA_SUB, load.len - t0);
                    const uint32_t at = n > 0 ? (uint32_t)page[sub] : 0u, behind = n > 0 ? (uint32_t)slot : 0u;
                    const char* kp = k_base + at * k_page + behind * k_token;
                    const char* vp = v_base + at * v_page + behind * v_token;
                    if (lane == 0) s_mask[warp][load_stage][sub] = (1u << n) - 1u;
                    if (n == PA_SUB && chunk_in) {
                        // (a stage begins at a multiple of a row's bytes, and rows i ROWS_PER_LOAD + row0 differ from row0 in
                        // other bits of the swizzle only; tokens that lie together need no address arithmetic)
                        if (p.k_token == D && p.v_token == D) {
#pragma unroll
                            for (int i = 0; i < LOADS; ++i) {
                                const uint32_t to = ((base + to0) ^ ((i * ROWS_PER_LOAD & 7) << 4)) + i * ROWS_PER_LOAD * (D * 2);
                                pa_cp_async(to, kp + i * ROWS_PER_LOAD * D * 2, true);
                                pa_cp_async(to + PA_SUB * D * 2, vp + i * ROWS_PER_LOAD * D * 2, true);
                            }
                        } else {
                            const uint32_t k_step = ROWS_PER_LOAD * k_token, v_step = ROWS_PER_LOAD * v_token;
#pragma unroll
                            for (int i = 0; i < LOADS; ++i) {
                                const uint32_t to = ((base + to0) ^ ((i * ROWS_PER_LOAD & 7) << 4)) + i * ROWS_PER_LOAD * (D * 2);
                                pa_cp_async(to, kp, true);
                                pa_cp_async(to + PA_SUB * D * 2, vp, true);
                                kp += k_step;
                                vp += v_step;
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < LOADS; ++i) {
                            const int row = i * ROWS_PER_LOAD + row0;
                            const bool read = chunk_in && row < n;
                            const uint32_t to = base + row * (D * 2) + ((chunk ^ (row & 7)) << 4);
                            pa_cp_async(to, read ? kp + i * ROWS_PER_LOAD * k_token : reinterpret_cast<const char*>(p.k), read);
                            pa_cp_async(to + PA_SUB * D * 2, read ? vp + i * ROWS_PER_LOAD * v_token : reinterpret_cast<const char*>(p.v), read);
                        }
                    }
                } else {
                    const int32_t t = t0 + (lane & 15), slot = t - page_number(t) * p.page_size;
                    const bool in = page[sub] >= 0;
                    const int64_t k_off = in ? page[sub] * p.k_page + load.head * p.k_head + slot * p.k_token : 0;
                    const int64_t v_off = in ? page[sub] * p.v_page + load.head * p.v_head + slot * p.v_token : 0;
                    const uint32_t mask = __ballot_sync(FULL_MASK, in) & 0xFFFFu;
                    if (lane == 0) s_mask[warp][load_stage][sub] = mask;
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) {
                        const int row = i * ROWS_PER_LOAD + row0;
                        const int64_t ko = __shfl_sync(FULL_MASK, k_off, row), vo = __shfl_sync(FULL_MASK, v_off, row);
                        const bool read = chunk_in && (mask >> row & 1);
                        const uint32_t to = base + row * (D * 2) + ((chunk ^ (row & 7)) << 4);
                        pa_cp_async(to, reinterpret_cast<const T*>(p.k) + ko + (read ? chunk * 8 : 0), read);
                        pa_cp_async(to + PA_SUB * D * 2, reinterpret_cast<const T*>(p.v) + vo + (read ? chunk * 8 : 0), read);
                    }
                }
            }
            ++loaded;
            load.next(p);
            if (loaded < count) {
                if (load.tile == 0) {                                         // a stream begins: its queries will be wanted
                    new_stream();
                    if (lane < load.heads(p))
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const T*>(p.q) + load.seq * p.q_seq + (load.first_head(p) + lane) * p.q_head));
                }
#pragma unroll
                for (int sub = 0; sub < SUBS; ++sub) page[sub] = page_of(load, sub);          // ready by the next call
            }
        }
        pa_cp_commit();
        load_stage = load_stage + 1 == STAGES ? 0 : load_stage + 1;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) load_tile();

    // where the lane's rows of the matrices lie in a stage: tokens lane & 15 of the keys, (lane & 7) + 8 (lane >> 4) of the values
    const uint32_t k_lane = (lane & 15) * (D * 2) + (((lane >> 4) ^ (lane & 7)) << 4);
    const uint32_t v_lane = ((lane & 7) + ((lane >> 4) << 3)) * (D * 2) + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
    const float far = PaWeights<T>::LAG / c;                                  // how far the reference of the exponents may lag the maximum
    uint32_t qf[N8][KSTEPS][2];
    // of heads 8 n + 2 quad and + 1.  The sums of weights are compensated: a lane that holds a sink would round thousands of
    // small weights to its sum's 2^-24 (14000 tokens 2^-25 below: lse off by 4e-5)
    float o[MT][N8][4], m[N8][2], l[N8][2], l_over[N8][2];
    bool fresh = true, whole = work.tile == 0;                                // a new stream begins / it began in this share
    int stage = 0;
    if (!whole) share.first = work.heads(p);
    for (uint32_t done = 0; done < count; ++done) {
        load_tile();
        if (fresh) {
            fresh = false;
            const int32_t head0 = work.first_head(p), rows = work.heads(p);
            const T* q = reinterpret_cast<const T*>(p.q) + work.seq * p.q_seq + head0 * p.q_head;
#pragma unroll
            for (int n = 0; n < N8; ++n) {
                m[n][0] = m[n][1] = LOWEST;
                l[n][0] = l[n][1] = l_over[n][0] = l_over[n][1] = 0.f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int r = n * 8 + g, col = ks * 16 + i * 8 + quad * 2;
                        qf[n][ks][i] = r < rows && col < p.dim ? *reinterpret_cast<const uint32_t*>(q + r * p.q_head + col) : 0u;
                    }
            }
        }
        pa_cp_wait<STAGES - 1>();
        __syncwarp();
        const uint32_t kb = ring + stage * Shape::STAGE_BYTES, vb = kb + PA_SUB * D * 2;
        // scores: 16 tokens x 8 N8 heads a step (a stage begins at a multiple of a row's bytes, so that 32 dimensions on is
        // an exclusive or); two chains of products, for their latency
        float s[SUBS][N8][4];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            float even[N8][4] = {}, odd[N8][4] = {};
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ks += 2) {
                uint32_t a[4], b[4];
                pa_ldmatrix(a, (kb + sub * Shape::SUB_BYTES + k_lane) ^ (ks << 5));
                pa_ldmatrix(b, (kb + sub * Shape::SUB_BYTES + k_lane) ^ ((ks + 1) << 5));
#pragma unroll
                for (int n = 0; n < N8; ++n) {
                    pa_mma<T>(even[n], a, qf[n][ks][0], qf[n][ks][1]);
                    pa_mma<T>(odd[n], b, qf[n][ks + 1][0], qf[n][ks + 1][1]);
                }
            }
            const uint32_t mask = s_mask[warp][stage][sub];
#pragma unroll
            for (int n = 0; n < N8; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[sub][n][i] = even[n][i] + odd[n][i];
            if (mask != 0xFFFFu) {
#pragma unroll
                for (int n = 0; n < N8; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(mask >> (g + (i >> 1) * 8) & 1)) s[sub][n][i] = -INFINITY;
            }
        }
        // running maxima of the thread's heads (i & 1), over its tokens and the eight lanes of the same quad
        float top[N8][2];
        bool higher = false;
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float t = fmaxf(s[0][n][h], s[0][n][2 + h]);
#pragma unroll
                for (int sub = 1; sub < SUBS; ++sub) t = fmaxf(t, fmaxf(s[sub][n][h], s[sub][n][2 + h]));
                t = fmaxf(t, __shfl_xor_sync(FULL_MASK, t, 4));
                t = fmaxf(t, __shfl_xor_sync(FULL_MASK, t, 8));
                t = fmaxf(t, __shfl_xor_sync(FULL_MASK, t, 16));
                top[n][h] = t;
                higher = higher || t > m[n][h] + far;
            }
        if (__any_sync(FULL_MASK, higher)) {                                  // (rare after a stream's first tile)
#pragma unroll
            for (int n = 0; n < N8; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float to = fmaxf(m[n][h], top[n][h]), f = exp2_approx((m[n][h] - to) * c);
                    m[n][h] = to;
                    l[n][h] *= f;
                    l_over[n][h] *= f;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) { o[mt][n][h] *= f; o[mt][n][2 + h] *= f; }
                }
        }
        // The probabilities enter the second product as two numbers of the cache's type, the rounded one and what the
        // rounding left off: one alone would add an error as large as the rounding of the output.
        uint32_t hi[SUBS][N8][2], lo[SUBS][N8][2];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int n = 0; n < N8; ++n) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = exp2_approx(fmaf(s[sub][n][i] - m[n][i & 1], c, PaWeights<T>::SHIFT));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float add = e[h] + e[2 + h] - l_over[n][h], to = l[n][h] + add;
                    l_over[n][h] = (to - l[n][h]) - add;
                    l[n][h] = to;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t w = pa_pack<T>(e[2 * i], e[2 * i + 1]);
                    const float2 r = pa_unpack<T>(w);
                    hi[sub][n][i] = pa_transpose(w);
                    lo[sub][n][i] = pa_transpose(pa_pack<T>(e[2 * i] - r.x, e[2 * i + 1] - r.y));
                }
            }
        // A tile's products are summed by themselves and then added: the matrix unit cuts off what lies below its accumulator's
        // last bit, which beside a sink's value would be a part of every further tile (14000 tokens: 2^-13 of the output).
#pragma unroll
        for (int m0 = 0; m0 < MT; m0 += AT_ONCE) {
            float acc[AT_ONCE][N8][4] = {};
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                uint32_t a[AT_ONCE][4];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) pa_ldmatrix_trans(a[i], (vb + sub * Shape::SUB_BYTES + v_lane) ^ ((m0 + i) << 5));
#pragma unroll
                for (int n = 0; n < N8; ++n) {
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i) pa_mma<T>(acc[i][n], a[i], hi[sub][n][0], hi[sub][n][1]);
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i) pa_mma<T>(acc[i][n], a[i], lo[sub][n][0], lo[sub][n][1]);
                }
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                for (int n = 0; n < N8; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[m0 + i][n][j] += acc[i][n][j];
        }
        __syncwarp();                                                         // the stage may be filled again
        stage = stage + 1 == STAGES ? 0 : stage + 1;

        const bool stream_ends = work.tile + 1 == work.tiles;
        if (stream_ends || done + 1 == count) {
            const bool final = whole && stream_ends;
            const int32_t head0 = work.first_head(p), rows = work.heads(p);
            const int64_t out_row = (int64_t)work.seq * p.heads + head0;
            float* part = slots + (2 * warp + (whole ? 1 : 0)) * Shape::SLOT;
#pragma unroll
            for (int n = 0; n < N8; ++n) {
                float inv[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float sum = l[n][h];
                    sum += __shfl_xor_sync(FULL_MASK, sum, 4);
                    sum += __shfl_xor_sync(FULL_MASK, sum, 8);
                    sum += __shfl_xor_sync(FULL_MASK, sum, 16);
                    inv[h] = sum == 0.f ? 0.f : 1.f / sum;                    // nothing held a token: zeros
                    const int row = n * 8 + quad * 2 + h;
                    if (g == 0 && row < rows) {
                        if (final) p.lse[out_row + row] = pa_lse<T>(m[n][h], sum, p.scale);
                        else { s_max[warp][whole ? 1 : 0][row] = m[n][h]; s_sum[warp][whole ? 1 : 0][row] = sum; }
                    }
                }
                if (final) {
                    // rows of the transposed matrix are heads: lane 4 g + quad gets dimensions 2 quad and + 1 of head 8 n + g
                    T* out = reinterpret_cast<T*>(p.out) + (out_row + n * 8 + g) * p.dim;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t w = pa_transpose(pa_pack<T>(o[mt][n][2 * i] * inv[0], o[mt][n][2 * i + 1] * inv[1]));
                            const int at = mt * 16 + i * 8 + quad * 2;
                            if (n * 8 + g < rows && at < p.dim) *reinterpret_cast<uint32_t*>(out + at) = w;
                        }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = n * 8 + quad * 2 + h;
                        if (row < rows)
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                part[row * D + mt * 16 + g] = o[mt][n][h];
                                part[row * D + mt * 16 + 8 + g] = o[mt][n][2 + h];
                            }
                    }
                }
            }
            if (!whole) share.first_ends = stream_ends;
            if (whole && !stream_ends) {
                const long long end = u0 + done + (work.tiles - work.tile);   // the first unit behind the stream
                share.seq = work.seq;
                share.head = head0;
                share.heads = rows;
                share.last = shares.of(end - 1);
            }
            fresh = whole = true;
        }
        work.next(p);
        if ((done + 1) % PA_PACE == 0 && turn < turns) {
            ++turn;
            __syncthreads();
        }
    }
    pa_cp_wait<0>();
    }
    for (; turn < turns; ++turn) __syncthreads();
    // sequences without tokens
    for (int32_t s = blockIdx.x; s < p.seqs; s += gridDim.x) {
        if (pa_length(p, s) > 0) continue;
        T* o = reinterpret_cast<T*>(p.out) + (int64_t)s * p.heads * p.dim;
        for (int32_t i = tid; i < p.heads * p.dim; i += THREADS) o[i] = Logit<T>::from_float(0.f);
        for (int32_t i = tid; i < p.heads; i += THREADS) p.lse[(int64_t)s * p.heads + i] = -INFINITY;
    }
    // The parts of the CTA's warps, chain by chain: a chain begins with a stream that goes on behind a warp's share, or with
    // the CTA's first stream where that began in an earlier CTA; it is an output if it lies within the CTA, else a part.
    if (lane == 0) s_share[warp] = share;
    __syncthreads();
    // (every thread makes the list of chains; the work on all of them is then one loop)
    PaMeta meta{-1, 0, 0, 0};
    int32_t from = -1, heads = 0, last = -1;                                  // the chain's first warp (-1: no chain), heads, last warp
    bool inside = false;                                                      // it began in this CTA
    int32_t before = 0, chains = 0;
    auto close = [&](bool ends) {
        if (tid == 0) s_chain[chains] = PaChain{from, last, heads, before, inside, inside && ends};
        before += heads;
        ++chains;
        from = -1;
    };
    for (int w = 0; w < WARPS; ++w) {
        const PaShare s = s_share[w];
        if (s.first > 0) {
            if (from < 0) { from = w; heads = s.first; inside = false; }
            last = w;
            if (s.first_ends) close(true);
        }
        if (s.heads > 0) { from = last = w; heads = s.heads; inside = true; }
    }
    if (from >= 0) {
        if (inside) meta = PaMeta{s_share[from].seq, s_share[from].head, s_share[from].heads, s_share[from].last / WARPS};
        close(false);
    }
    if (tid == 0) p.meta[blockIdx.x] = meta;
    __syncthreads();
    int chain = 0;
    for (int32_t i = tid; i < before * (D / 4); i += THREADS) {
        const int32_t at = i % (D / 4) * 4;
        while (chain + 1 < chains && i / (D / 4) >= s_chain[chain + 1].before) ++chain;
        const PaChain k = s_chain[chain];
        const int32_t row = i / (D / 4) - k.before;
        float top = LOWEST, sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = k.from; w <= k.last; ++w) top = fmaxf(top, s_max[w][k.inside && w == k.from][row]);
#pragma unroll 4
        for (int w = k.from; w <= k.last; ++w) {
            const int which = k.inside && w == k.from;
            const float f = exp2_approx((s_max[w][which][row] - top) * c);
            const float4 x = *reinterpret_cast<const float4*>(slots + (2 * w + which) * Shape::SLOT + row * D + at);
            sum = fmaf(f, s_sum[w][which][row], sum);
            acc.x = fmaf(f, x.x, acc.x);
            acc.y = fmaf(f, x.y, acc.y);
            acc.z = fmaf(f, x.z, acc.z);
            acc.w = fmaf(f, x.w, acc.w);
        }
        if (k.final) {
            const int64_t out_row = (int64_t)s_share[k.from].seq * p.heads + s_share[k.from].head + row;
            if (at < p.dim) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                const uint2 w2 = make_uint2(pa_pack<T>(acc.x * inv, acc.y * inv), pa_pack<T>(acc.z * inv, acc.w * inv));
                *reinterpret_cast<uint2*>(reinterpret_cast<T*>(p.out) + out_row * p.dim + at) = w2;
            }
            if (at == 0) p.lse[out_row] = pa_lse<T>(top, sum, p.scale);
        } else {
            float* part = slots + (2 * WARPS + (k.inside ? 1 : 0)) * Shape::SLOT;
            *reinterpret_cast<float4*>(part + row * D + at) = acc;
            if (at == 0) { part[PA_ROWS * D + row] = top; part[PA_ROWS * (D + 1) + row] = sum; }
        }
    }
}

// Joins the parts of a stream that several CTAs share, one warp per head; where they are many, one CTA per head.
// grid: (CTAs of the first kernel, heads per pass).
constexpr int PJ_THREADS = 128;
// More parts than this are split among a CTA's warps: one sequence of 131072 tokens and one key-value head, 148 parts, 25.0 us,
// with a warp for all of a head's parts 33.8.
constexpr int PJ_MANY = 16;
template <typename T, int D>
__global__ void __launch_bounds__(PJ_THREADS) paged_attention_join_kernel(const PaParams p) {
    using Shape = PaShape<D>;
    constexpr int WARPS = PJ_THREADS / 32, COLS = D / 32;                     // columns per lane: 2, 4 or 8
    __shared__ __align__(16) float s_acc[WARPS][D];
    __shared__ float s_sum[WARPS], s_top[WARPS];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t first = blockIdx.x;
    auto slot = [&](int32_t i) { return p.parts + ((int64_t)(first + i) * Shape::SLOTS + 2 * Shape::WARPS + (i == 0 ? 1 : 0)) * Shape::SLOT; };
    const float c = p.scale * LOG2E;
    float top = LOWEST, sum = 0.f, acc[COLS];
#pragma unroll
    for (int j = 0; j < COLS; ++j) acc[j] = 0.f;
    struct Part { float m, l, o[COLS]; };
    auto read = [&](int32_t i, int32_t row) {
        const float* s = slot(i);
        Part x;
        x.m = s[PA_ROWS * D + row];
        x.l = s[PA_ROWS * (D + 1) + row];
#pragma unroll
        for (int j = 0; j < COLS; ++j) x.o[j] = s[row * D + j * 32 + lane];
        return x;
    };
    auto add = [&](const Part& x) {
        const float to = fmaxf(top, x.m), f = exp2_approx((top - to) * c), e = exp2_approx((x.m - to) * c);
        top = to;
        sum = fmaf(e, x.l, f * sum);
#pragma unroll
        for (int j = 0; j < COLS; ++j) acc[j] = fmaf(e, x.o[j], f * acc[j]);
    };
    // Most streams have two parts, this CTA's and the next one's: they are read along with what says so (and thrown away if
    // it does not; scratch memory holds them in any case).
    const int guess = (int)blockIdx.y * WARPS + warp;
    Part own, next;
    const bool guessed = guess < p.rows && first + 1 < (int32_t)gridDim.x;
    if (guessed) { own = read(0, guess); next = read(1, guess); }
    const PaMeta meta = p.meta[blockIdx.x];
    if (meta.seq < 0) return;
    const int32_t n = meta.last - first + 1;
    const bool many = n > PJ_MANY;
    const int row = many ? (int)blockIdx.y : guess;
    if (row >= meta.heads) return;                                            // (many: the whole CTA)
    auto add_all = [&](int32_t begin, int32_t step) {                         // eight parts' loads in flight at a time
        constexpr int AT_ONCE = D == 256 ? 4 : 8;
        for (int32_t i0 = begin; i0 < n; i0 += AT_ONCE * step) {
            Part x[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (i0 + u * step < n) x[u] = read(i0 + u * step, row);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (i0 + u * step < n) add(x[u]);
        }
    };
    if (!many) {
        add(own);                                                             // (two parts at least, so that they were read)
        add(next);
        add_all(2, 1);
    } else {
        add_all(warp, WARPS);
    }
    if (many) {
#pragma unroll
        for (int j = 0; j < COLS; ++j) s_acc[warp][j * 32 + lane] = acc[j];
        if (lane == 0) { s_sum[warp] = sum; s_top[warp] = top; }
        __syncthreads();
        if (warp > 0) return;
        top = LOWEST;
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < COLS; ++j) acc[j] = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            Part x;
            x.m = s_top[w];
            x.l = s_sum[w];
#pragma unroll
            for (int j = 0; j < COLS; ++j) x.o[j] = s_acc[w][j * 32 + lane];
            add(x);
        }
    }
    const int64_t out_row = (int64_t)meta.seq * p.heads + meta.head + row;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T* out = reinterpret_cast<T*>(p.out) + out_row * p.dim;
#pragma unroll
    for (int j = 0; j < COLS; ++j)
        if (j * 32 + lane < p.dim) out[j * 32 + lane] = Logit<T>::from_float(acc[j] * inv);
    if (lane == 0) p.lse[out_row] = pa_lse<T>(top, sum, p.scale);
}

}  // namespace profk
