// Attention of a chunk of new tokens of every sequence over a paged key-value cache that holds them already:
//   out_h = sum_j p_j v_j,   p = softmax_j(scale q_h . k_j),   lse_h = ln sum_j e^(scale q_h . k_j),
// for the new token at place t of its sequence over the tokens j <= t.
//
// Prompts are bound by the matrix unit (4 dim operations per query head, new token and seen key), drafts of a few tokens by
// HBM.  Query heads that share a key-value head are rows of the same tile: row r of a (sequence, key-value head) is the
// token r / group and the head r % group, so that the cache is read once for all of them.
//
// A CTA has an SM to itself.  Two streams of 128 rows (two tiles of queries over every tile of keys; or, where there are no
// more than 128 rows, one tile of queries whose tiles of keys alternate between the streams) take turns on the matrix unit:
// while one stream's scores are turned into weights by its four warps, the other's products run.
//   S = Q K^T   tcgen05.mma, both operands in shared memory, S in tensor memory;
//   P           a thread owns a row: reads its scores, keeps the running maximum and sum, writes the weights over the scores;
//   O += P V    tcgen05.mma, P from tensor memory, V from shared memory as it was loaded (its rows run along the product).
// With dim > 128 there is room for one O only: one stream, whose scores alternate between two places.
// The exponents' reference is raised only when a score passes it by more than 2^8 (fp16: 2^4; its weights are lifted by 2^11 so
// that small ones do not vanish); then the row's own thread scales its O.  Weights are rounded once to the cache's type, as the
// product with the values needs it: each is off by half a step at most (bf16: 2^-8 of itself; fp16: 2^-11, or 2^-36 of the largest).  For
// values of either sign that adds up to about as much as the rounding of the output does (root mean squares over the outputs against 64
// bits: 1.1 to 1.4 times what fp32 weights give); a row with nearly all its weight on one token carries that token's error as a factor.
// (Two numbers to a weight, as in the form for one token, would be twice the products with the values.)  Sums of weights are kept in
// fp32, unrounded and compensated: lse has no part in that rounding.
//
// The work is the list of (sequence, key-value head, block of rows, tile of keys), cut into one contiguous share per CTA by
// cost whatever the lengths; items that a cut goes through leave unnormalised parts, which a second kernel joins in order.
//
// Measured: 2 x 2048 tokens behind 65536 and 129024, 32 heads of 128 on 8, bf16: 5.6 ms on a cold device (1.15 PFLOP/s), 6.4 to 7.5 in a
// loop, where power sets the clock; a stream's tile takes 3500 cycles, of which its weights 2050, its products 1024, the rest
// hands over.  32 sequences of 1 to 8192 tokens with four drafts, 64 heads on 8: 134 to 140 us, device by device, for 82 us of HBM.
// 24 ragged prompts of 1 to 2500 tokens, 16 heads of 64, fp16: 317 us.  One prompt of 301 tokens: 19 us.
#pragma once

#include <cuda.h>

#include <cstddef>

#include "logits.cuh"

namespace profk {

constexpr int CA_ROWS = 128;              // rows of a tile of queries: lanes of the tensor memory
constexpr int CA_THREADS = 384;           // two warpgroups of weights; three warps that load, one that issues products
constexpr int CA_LOADERS = 96, CA_LOAD_ROWS = CA_LOADERS / 8;            // eight threads to 128 bytes of a row
constexpr int CA_OVERHEAD = 3;            // what an item costs beside its tiles, in units of one tile of one stream (in turn on one device: 2: drafts 133 us, ragged prompts 327; 3: 134, 317; 5: 136, 320)
constexpr int CA_MASKS = 8;               // tiles whose masks are kept; loading runs ahead by fewer
constexpr int CA_ITEMS = 4;               // items whose bad tokens are kept
constexpr int CA_BAD_TILES = 4;           // tiles of an item that its mask can cut
constexpr int CA_POLLS = 1 << 22;
constexpr int CA_MANY_REGISTERS = 208, CA_FEW_REGISTERS = 88;      // of a thread that weighs, and of the others, after the launch

template <int D>
struct CaShape {
    static constexpr int STREAMS = D <= 128 ? 2 : 1;
    static constexpr int KT = D <= 128 ? 128 : 64;                       // tokens of a tile
    static constexpr int BLOCK = STREAMS * CA_ROWS;                      // rows of an item
    static constexpr int Q_TILE = CA_ROWS * D * 2, STAGE = KT * D * 2;
    static constexpr int STAGES = D == 64 ? 8 : 5;
    static constexpr int O_AT = 256;                                     // columns of the tensor memory: S 0 and 128, O from here
};

// n / d for n < 2^31 by a multiplication: m = ceil(2^(31 + l) / d), l = ceil(log2 d), and n m >> (31 + l).
struct CaDivisor {
    uint32_t d, m, shift;                 // shift: l - 1; d = 1 has none
    __host__ static CaDivisor of(uint32_t d) {
        uint32_t l = 0;
        while ((1ull << l) < d) ++l;
        return {d, d == 1 ? 0u : (uint32_t)(((1ull << (31 + l)) + d - 1) / d), l - 1};
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return d == 1 ? n : __umulhi(n, m) >> shift; }
};

// Descriptions of keys, values (dim, token of a page, head, page) and queries (dim, head, token, sequence) for tiled copies.
struct CaMaps { CUtensorMap k, v, q; };

template <typename T>
struct CaParams {
    const T* q;
    int64_t q_seq, q_token, q_head;       // strides in elements
    const T* k;
    const T* v;
    int64_t ks_page, ks_head, ks_token, vs_page, vs_head, vs_token;
    const int32_t* tables;
    int64_t table_stride;
    const int32_t* lengths;
    const int32_t* starts;                // null: `tokens` rows each
    int32_t rows, tokens;
    int32_t seqs, heads, kv_heads, group, dim, page_size, pages, width;
    CaDivisor by_group, by_page;
    int32_t box;                          // tokens of one tiled copy: they never leave a page; 0: tokens are copied one by one
    bool q_box;                           // queries are copied by tile, too
    bool q_wide;                          // rows of q lie on 16-byte vectors
    float scale;
    int32_t polls;                        // that a wait may take: CA_POLLS but for tests
    T* out;
    float* lse;
    float* parts;                         // (2 per CTA) x BLOCK x D
    float2* sums;                         // (2 per CTA) x BLOCK: reference, sum
    struct CaMeta* meta;                  // 2 per CTA
};

struct CaMeta {
    int32_t valid, last, failed, rows;    // of this part: whether there is one, whether it ends its item
    int32_t row0;                         // of the first new token, in q and out
    int32_t head, first;                  // key-value head; first row of the item
};

// ---- items -------------------------------------------------------------------------------------

// The new tokens of a sequence: first row, how many, place of the first.  (Rows times heads stay below 2^31.  A place below
// -2^31 is taken for that: all tokens of such a sequence lie before its beginning.)
struct CaSeq { int32_t row0, n, base; };
template <typename T>
__device__ __forceinline__ CaSeq ca_seq(const CaParams<T>& p, int32_t s) {
    CaSeq q;
    if (p.starts) {
        q.row0 = max(0, min(p.starts[s], p.rows));
        q.n = max(q.row0, min(p.starts[s + 1], p.rows)) - q.row0;
    } else {
        q.row0 = s * p.tokens;
        q.n = p.tokens;
    }
    q.base = (int32_t)max((int64_t)p.lengths[s] - q.n, (int64_t)INT32_MIN);
    return q;
}

// Block b of a sequence's rows: its first row, how many; tokens that its last row sees, tiles of them; a tile's weight.
template <int D>
struct CaBlock {
    int32_t first, rows, end, tiles;
    __device__ __forceinline__ CaBlock(const CaSeq& s, const CaDivisor& group, int32_t room, int32_t b) {
        using S = CaShape<D>;
        first = b * S::BLOCK;
        rows = min(S::BLOCK, s.n * (int32_t)group.d - first);
        end = (int32_t)max(0ll, min((long long)s.base + group.quotient((uint32_t)(first + rows - 1)) + 1, (long long)room));
        tiles = (int32_t)(((uint32_t)end + S::KT - 1) / S::KT);
    }
    __device__ __forceinline__ int32_t weight() const { return rows > CA_ROWS ? 2 : 1; }
    __device__ __forceinline__ int32_t cost() const { return CA_OVERHEAD + weight() * tiles; }
    // tiles in front of unit x of the item
    __device__ __forceinline__ int32_t tile_of(int32_t x) const { return x <= CA_OVERHEAD ? 0 : min(tiles, (x - CA_OVERHEAD + weight() - 1) / weight()); }
};
template <int D>
__device__ __forceinline__ int32_t ca_blocks(const CaSeq& s, int32_t group) { return (int32_t)(((uint32_t)(s.n * group) + CaShape<D>::BLOCK - 1) / CaShape<D>::BLOCK); }
template <int D>
__device__ __forceinline__ int64_t ca_head_cost(const CaSeq& s, const CaDivisor& group, int32_t room) {
    int64_t sum = 0;
    for (int32_t b = 0, n = ca_blocks<D>(s, (int32_t)group.d); b < n; ++b) sum += CaBlock<D>(s, group, room, b).cost();
    return sum;
}

struct CaPlace {                          // an item, and its first unit
    int64_t at;
    int32_t block, seq, head;
};

// What a share covers, item by item; every warp walks by itself.
template <typename T, int D>
struct CaWalk {
    const CaParams<T>& p;
    int64_t left;                         // units from the item's first to the share's end
    int32_t skip;                         // units of the item in front of the share
    int32_t block_number, seq_number, head;
    CaSeq seq;
    int32_t number = -1;                  // of the item, among those with tiles
    bool begun = false;
    // the item:
    CaBlock<D> block;
    int32_t tile0, tile1;
    __device__ __forceinline__ CaWalk(const CaParams<T>& params, const CaPlace& start, int64_t from, int64_t to)
        : p(params), left(from < to ? to - start.at : 0), skip(from < to ? (int32_t)(from - start.at) : 0), block_number(start.block), seq_number(start.seq),
          head(start.head), seq(ca_seq(params, from < to ? start.seq : 0)), block(seq, params.by_group, room(), from < to ? start.block : 0), tile0(0), tile1(0) {}
    __device__ __forceinline__ int32_t room() const { return p.width * p.page_size; }
    __device__ __forceinline__ bool next() {
        for (;;) {
            if (begun) {
                left -= block.cost();
                skip -= block.cost();
                if (left <= 0) return false;
                if (++block_number >= ca_blocks<D>(seq, p.group)) {
                    block_number = 0;
                    if (++head >= p.kv_heads) {
                        head = 0;
                        do {
                            if (++seq_number >= p.seqs) return false;
                            seq = ca_seq(p, seq_number);
                        } while (seq.n == 0);
                    }
                }
                block = CaBlock<D>(seq, p.by_group, room(), block_number);
            } else {
                if (left <= 0) return false;
                begun = true;
            }
            tile0 = block.tile_of(max(skip, 0));
            tile1 = block.tile_of((int32_t)min(left, (int64_t)block.cost()));
            if (tile1 > tile0 || (block.tiles == 0 && skip <= 0)) {
                number += tile1 > tile0;
                return true;
            }
        }
    }
    __device__ __forceinline__ bool whole() const { return tile0 == 0 && tile1 == block.tiles; }
};

// ---- instructions ------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t ca_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// Barriers, by their addresses in shared memory.
__device__ __forceinline__ void ca_bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void ca_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Whether a phase has passed, at once; and likewise after the hardware has waited for it a while.
__device__ __forceinline__ bool ca_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool ca_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// A warp waits for a phase; gives up after a limit (the word behind `failed`: 0 for what is not over at once), or when another warp has,
// and then returns false for good.
__device__ __forceinline__ bool ca_wait(uint32_t bar, uint32_t parity, volatile int32_t* failed) {
    if (__all_sync(FULL_MASK, ca_test(bar, parity))) return true;
    int32_t left = failed[1];
#pragma unroll 1
    while (!__any_sync(FULL_MASK, failed[0] != 0 || left-- <= 0)) {
        if (__all_sync(FULL_MASK, ca_try(bar, parity))) return true;
    }
    failed[0] = 1;
    return false;
}
// Waits for what is still under way in the CTA's memory, before that is given up and whatever has failed; limited, too.
__device__ __forceinline__ void ca_drain(uint32_t bar, uint32_t parity) {
    int32_t left = CA_POLLS;
#pragma unroll 1
    while (!__all_sync(FULL_MASK, ca_try(bar, parity)) && --left > 0) {}
}
// Warps meet (the barrier counts them); the wait is limited as all others are.
__device__ __forceinline__ bool ca_meet(uint32_t bar, uint32_t& phase, volatile int32_t* failed) {
    __syncwarp();
    if ((threadIdx.x & 31u) == 0) ca_arrive(bar);
    const bool ok = ca_wait(bar, phase, failed);
    phase ^= 1u;
    return ok;
}

__device__ __forceinline__ void ca_commit(uint32_t bar, uint32_t one) {
    asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(one) : "memory");
}
__device__ __forceinline__ void ca_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void ca_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A value that all lanes hold alike, told to the compiler: the matrix instructions take their operands from uniform registers.
__device__ __forceinline__ uint32_t ca_uniform(uint32_t x) { return __shfl_sync(FULL_MASK, x, 0); }
__device__ __forceinline__ uint32_t ca_elect() {
    uint32_t one;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one;
}
// D (128 x N, tensor memory) (+)= A (shared memory or tensor memory) B (shared memory), issued by the lane whose `one` is set.
// (A predicate, not a branch: in diverged code the operands may be computed in ordinary registers and moved one by one, which
// made the whole kernel 40 % slower.)
__device__ __forceinline__ void ca_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add, uint32_t one) {
    asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add), "r"(one) : "memory");
}
__device__ __forceinline__ void ca_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add, uint32_t one) {
    asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(what), "r"((uint32_t)add), "r"(one) : "memory");
}
// Shared-memory operand in rows of 128 bytes, swizzled in atoms of eight rows; `leading`: between atoms along a transposed
// operand's rows.  Its lower word holds what differs between operands: the address in 16 bytes (and `leading`).
__device__ __forceinline__ uint32_t ca_operand_low(uint32_t addr, uint32_t leading) { return (addr & 0x3FFFFu) >> 4 | leading >> 4 << 16; }
__device__ __forceinline__ uint64_t ca_operand(uint32_t low) { return (uint64_t)(1024u >> 4 | 1u << 14 | 2u << 29) << 32 | low; }
template <typename T> struct CaType;
template <> struct CaType<__nv_bfloat16> {
    static constexpr uint32_t CODE = 1;
    static constexpr float RAISE = 8.0f, LIFT = 0.0f;
    static constexpr uint32_t EXPONENT = 0x7F80u;
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <> struct CaType<__half> {
    static constexpr uint32_t CODE = 0;
    static constexpr float RAISE = 4.0f, LIFT = 11.0f;
    static constexpr uint32_t EXPONENT = 0x7C00u;
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
// 128 x N product of 16-bit operands summed in fp32; `transposed`: B's rows run along the summation.
template <typename T>
__device__ __forceinline__ constexpr uint32_t ca_product(uint32_t n, bool transposed) {
    return 1u << 4 | CaType<T>::CODE << 7 | CaType<T>::CODE << 10 | (transposed ? 1u << 16 : 0u) | (n >> 3) << 17 | (128u >> 4) << 24;
}

__device__ __forceinline__ void ca_tm_load(uint32_t addr, float* r) {
    uint32_t* u = reinterpret_cast<uint32_t*>(r);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]),
                   "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]),
                   "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
                 : "r"(addr));
}
__device__ __forceinline__ void ca_tm_store(uint32_t addr, const uint32_t* u) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(u[0]),
                 "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]),
                 "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]),
                 "r"(u[30]), "r"(u[31]), "r"(addr)
                 : "memory");
}
// The loads have ended; their 32 registers pass through, so that nothing that uses them moves in front.
__device__ __forceinline__ void ca_tm_loaded(float* r) {
    uint32_t* u = reinterpret_cast<uint32_t*>(r);
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]), "+r"(u[10]), "+r"(u[11]), "+r"(u[12]),
                   "+r"(u[13]), "+r"(u[14]), "+r"(u[15]), "+r"(u[16]), "+r"(u[17]), "+r"(u[18]), "+r"(u[19]), "+r"(u[20]), "+r"(u[21]), "+r"(u[22]), "+r"(u[23]), "+r"(u[24]),
                   "+r"(u[25]), "+r"(u[26]), "+r"(u[27]), "+r"(u[28]), "+r"(u[29]), "+r"(u[30]), "+r"(u[31])
                 :: "memory");
}
__device__ __forceinline__ void ca_tm_store16(uint32_t addr, const uint32_t* u) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]),
                 "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ca_tm_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint4 ca_read(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// 16 bytes from global to shared memory; zeros where there is nothing to read.
__device__ __forceinline__ void ca_copy(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16u : 0u) : "memory");
}

// ---- shared memory -----------------------------------------------------------------------------

template <int D>
struct CaControl {
    uint64_t full[CaShape<D>::STAGES], empty[CaShape<D>::STAGES];
    uint64_t q_full, q_free, s_full[2], p_full[2], o_full[2], o_step, loaders, weighers, opened, asked, looked, drain;
    uint32_t tensor;                      // address of the tensor memory
    int32_t failed[2];                    // whether a wait has run out; polls that one may take
    int32_t table[2][CaShape<D>::KT];     // pages of two tiles' tokens; -1: nothing there
    alignas(16) uint32_t mask[CA_MASKS][4];        // which tokens of a tile are there
    uint32_t bad[CA_ITEMS][CA_BAD_TILES][4];       // tokens whose values are not finite, of the tiles that a mask cuts
    uint32_t any_bad[CA_ITEMS];
    float2 other[CA_ROWS];                // reference and sum of the second stream, where two share rows
    CaPlace place[2];
    int64_t bound[2];
    int64_t scan[CA_THREADS / 32];
};
// The address of a member of the control block at address `ctl`.
#define CA_AT(ctl, member) ((ctl) + (uint32_t)offsetof(CaControl<D>, member))
template <int D>
constexpr size_t ca_smem_bytes() { return CaShape<D>::STREAMS * CaShape<D>::Q_TILE + CaShape<D>::STAGES * CaShape<D>::STAGE + sizeof(CaControl<D>); }
static_assert(ca_smem_bytes<128>() <= 232448 && ca_smem_bytes<256>() <= 232448 && ca_smem_bytes<64>() <= 232448, "an SM's shared memory");

__device__ __forceinline__ int64_t ca_quotient(int64_t a, int64_t b) { return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b; }

// Units of all items, and the share of this CTA: [bound[0], bound[1]) of them, beginning at place[0].  A cut that would leave
// little of an item on either side is moved to the item's nearer end: parts cost their reading and writing (items of up to 4 + rows / 16
// units; 2 + rows / 32: one prompt of 301 tokens 24 us for 19; 8 + rows / 8: ragged prompts 327 us for 317).  Each half of the
// threads goes over all sequences and finds one of the two bounds.
template <typename T, int D>
__device__ __noinline__ void ca_plan(const CaParams<T>& p, CaControl<D>* ctl) {
    constexpr int HALF = CA_THREADS / 2;
    const int32_t room = p.width * p.page_size;
    const int32_t which = (int32_t)threadIdx.x / HALF, tid = (int32_t)threadIdx.x % HALF, lane = tid & 31, warp = (int32_t)threadIdx.x / 32;
    const int32_t per = (p.seqs + HALF - 1) / HALF, s0 = min(p.seqs, tid * per), s1 = min(p.seqs, s0 + per);
    int64_t mine = 0, one = 0;
    CaSeq seq{};
    for (int32_t s = s0; s < s1; ++s) {
        seq = ca_seq(p, s);
        one = ca_head_cost<D>(seq, p.by_group, room);
        mine += one * p.kv_heads;
    }
    int64_t upto = mine;
    for (int d = 1; d < 32; d *= 2) {
        const int64_t o = __shfl_up_sync(FULL_MASK, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) ctl->scan[warp] = upto;
    __syncthreads();
    int64_t total = 0, before = upto - mine;
    for (int w = 0; w < HALF / 32; ++w) {
        const int64_t x = ctl->scan[which * (HALF / 32) + w];
        if (w < warp - which * (HALF / 32)) before += x;
        total += x;
    }
    const int64_t shares = min((int64_t)gridDim.x, max((int64_t)1, total / 4));       // (a share within an item holds a tile at least)
    const int64_t c = (int64_t)blockIdx.x + which, each = ca_quotient(total, shares);
    const int64_t x = c >= shares ? total : each * c + ca_quotient((total - each * shares) * c, shares);
    if (tid == 0 && x >= total) ctl->bound[which] = total;
    if (x >= before && x < before + mine) {
        int64_t at = before;
        for (int32_t s = s0; s < s1; ++s) {
            if (per > 1) {
                seq = ca_seq(p, s);
                one = ca_head_cost<D>(seq, p.by_group, room);
            }
            if (x >= at + one * p.kv_heads) { at += one * p.kv_heads; continue; }
            const int32_t head = (int32_t)ca_quotient(x - at, one);
            CaPlace place{at + head * one, 0, s, head};
            for (;; ++place.block) {
                const CaBlock<D> b(seq, p.by_group, room, place.block);
                if (x >= place.at + b.cost()) { place.at += b.cost(); continue; }
                // x lies in this item
                int64_t cut = x;
                if (x > place.at && b.cost() <= 4 + b.rows / 16) cut = x - place.at < place.at + b.cost() - x ? place.at : place.at + b.cost();
                ctl->bound[which] = cut;
                ctl->place[which] = place;                   // (a cut at the item's end: the walk steps over it)
                break;
            }
            break;
        }
    }
    __syncthreads();
}

// ---- loading -----------------------------------------------------------------------------------

// What a loading thread has in flight: groups of copies, oldest first, each with the barrier that tells of it.
template <typename T, int D>
struct CaLoader {
    using S = CaShape<D>;
    static constexpr int DEPTH = 3;
    CaControl<D>* ctl;
    uint32_t bars, stages;                // shared memory
    uint32_t pending[DEPTH];
    int32_t check[DEPTH];                 // values to look through: stage | tile's number << 8 | item's << 16; -1: none
    int32_t count = 0;
    int32_t stage = 0;
    uint32_t phase = 1;                   // of `empty`: the first round waits for nothing
    // The oldest copies have landed, once no more than `newer` groups are in flight: look through them if asked, tell.
    __device__ __forceinline__ void retire(int32_t newer) {
        if (newer == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
        else if (newer == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (newer == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (check[0] >= 0) look_through(ctl, stages, check[0] & 255, check[0] >> 8 & 255, check[0] >> 16, (int32_t)threadIdx.x - 256);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane_id() == 0) ca_arrive(pending[0]);
#pragma unroll
        for (int i = 0; i + 1 < DEPTH; ++i) { pending[i] = pending[i + 1]; check[i] = check[i + 1]; }
        --count;
    }
    __device__ __forceinline__ void issued(uint32_t bar, int32_t what) {
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (count == DEPTH) retire(DEPTH);
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
            if (i == count) { pending[i] = bar; check[i] = what; }
        ++count;
    }
    // Waits until a barrier's phase has passed; what has landed meanwhile is told of.
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) {
        while (count > 0) {
            if (__all_sync(FULL_MASK, ca_test(bar, parity))) return true;
            retire(count - 1);
        }
        return ca_wait(bar, parity, ctl->failed);
    }
    __device__ __forceinline__ void flush() {
        while (count > 0) retire(count - 1);
    }
    static __device__ __forceinline__ uint32_t chunk_at(int32_t row, int32_t chunk, int32_t rows) {
        return (uint32_t)((chunk >> 3) * rows * 128 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
    }
    // Whether any of eight elements is infinite or NaN: a carry out of an exponent of ones.
    static __device__ __forceinline__ uint32_t carries(const uint4& v) {
        constexpr uint32_t E = CaType<T>::EXPONENT * 0x10001u, ONE = (CaType<T>::EXPONENT & -CaType<T>::EXPONENT) * 0x10001u;
        return (((v.x & E) + ONE) | ((v.y & E) + ONE) | ((v.z & E) + ONE) | ((v.w & E) + ONE)) & 0x80008000u;
    }
    // The part of a tile of values of thread t of 8 * ROWS: vectors that are not finite are taken out, and their tokens noted.
    // Its part is vector t % 8 of every ROWS-th row, in each 128-byte column.  Of the threads that copy (ROWS = CA_LOAD_ROWS) these are
    // the vectors that the thread copied itself: it has waited for no others.
    template <int ROWS>
    static __device__ __forceinline__ void look(CaControl<D>* ctl, uint32_t stages, int32_t st, int32_t tile, int32_t item, int32_t t) {
        const uint32_t at = stages + st * S::STAGE;
        uint32_t any = 0;
        if constexpr (ROWS % 8 == 0) {                                   // (a multiple of eight rows on, the swizzle is the same)
#pragma unroll 8
            for (int i = 0; i < S::KT * (D / 64); i += ROWS) any |= carries(ca_read(at + i * 128 + chunk_at(t >> 3, t & 7, S::KT)));
        } else {
#pragma unroll 256 / D
            for (int row = t >> 3; row < S::KT; row += ROWS) {
                const uint32_t first = at + chunk_at(row, t & 7, S::KT);
#pragma unroll
                for (int h = 0; h < D / 64; ++h) any |= carries(ca_read(first + h * (S::KT * 128)));
            }
        }
        if (any) take_out(ctl, at, tile, item, t, ROWS);
    }
    // (A call: few tiles need it.  In line its registers cost the 64-dimensional kernel 2 to 5 %, whatever the pages' size.)
    static __device__ __noinline__ void look_through(CaControl<D>* ctl, uint32_t stages, int32_t st, int32_t tile, int32_t item, int32_t t) {
        look<CA_LOAD_ROWS>(ctl, stages, st, tile, item, t);
    }
    static __device__ __noinline__ void take_out(CaControl<D>* ctl, uint32_t at, int32_t tile, int32_t item, int32_t t, int32_t rows_at_once) {
        const int32_t rounds = (S::KT + rows_at_once - 1) / rows_at_once;
#pragma unroll 1
        for (int i = 0; i < rounds * (D / 64); ++i) {
            const int32_t row = (t >> 3) + i % rounds * rows_at_once;
            if (row >= S::KT) continue;
            const uint32_t where = at + chunk_at(row, (t & 7) + i / rounds * 8, S::KT);
            if (!carries(ca_read(where))) continue;
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(where), "r"(0u) : "memory");
            atomicOr(&ctl->bad[item][tile][row / 32], 1u << (row % 32));
            ctl->any_bad[item] = 1;
        }
    }
    // One tile of keys or values.
    __device__ __forceinline__ bool tile(const CaParams<T>& p, const T* pages, int64_t page_stride, int64_t token_stride, int32_t buffer, int32_t first, int32_t what) {
        if (!wait(CA_AT(bars, empty) + stage * 8, phase)) return false;
        const int32_t t = (int32_t)threadIdx.x - 256;
        const uint32_t to = stages + stage * S::STAGE;
#pragma unroll 4
        for (int32_t row = t >> 3; row < S::KT; row += CA_LOAD_ROWS) {
            const int32_t page = ctl->table[buffer][row];
            const uint32_t token = (uint32_t)(first + row);
            const uint32_t slot = token - p.by_page.quotient(token) * p.by_page.d;
            const T* from = pages + max(page, 0) * page_stride + (page >= 0 ? slot * token_stride : 0);
#pragma unroll
            for (int h = 0; h < D / 64; ++h) {
                const int32_t chunk = (t & 7) + 8 * h;
                const bool there = page >= 0 && chunk * 8 < p.dim;
                ca_copy(to + chunk_at(row, chunk, S::KT), there ? from + chunk * 8 : pages, there);
            }
        }
        issued(CA_AT(bars, full) + stage * 8, what < 0 ? -1 : what | stage);
        if (++stage == S::STAGES) { stage = 0; phase ^= 1; }
        return true;
    }
};

// A thread's part of an item's queries: rows of (token, head), eight threads to 128 bytes.
template <typename T, int D>
__device__ __noinline__ void ca_copy_queries(const CaParams<T>& p, const CaWalk<T, D>& walk, uint32_t q_at, int32_t t, int32_t rows_at_once) {
    using S = CaShape<D>;
    const auto& b = walk.block;
    const T* q = p.q + (p.starts ? (int64_t)walk.seq.row0 * p.q_token : walk.seq_number * p.q_seq) + (int64_t)walk.head * p.group * p.q_head;
    const int32_t rows = b.rows > CA_ROWS ? 2 * CA_ROWS : CA_ROWS;
#pragma unroll 2
    for (int32_t r = t >> 3; r < rows; r += rows_at_once) {
        const bool held = r < b.rows;
        const uint32_t token = p.by_group.quotient((uint32_t)(b.first + r)), g = (uint32_t)(b.first + r) - token * p.group;
        const T* from = held ? q + token * p.q_token + g * p.q_head : p.q;
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
            const int32_t chunk = (t & 7) + 8 * h;
            const bool there = held && chunk * 8 < p.dim;
            const uint32_t to = q_at + r / CA_ROWS * S::Q_TILE + CaLoader<T, D>::chunk_at(r % CA_ROWS, chunk, CA_ROWS);
            if (p.q_wide) {
                ca_copy(to, there ? from + chunk * 8 : p.q, there);
            } else {
                uint32_t w[4] = {0, 0, 0, 0};
                if (there)
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(from)[chunk * 8 + e] << (16 * (e % 2));
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
            }
        }
    }
}
// The first tile of an item that some row does not see all of.
template <typename T, int D>
__device__ __forceinline__ int32_t ca_first_cut(const CaParams<T>& p, const CaWalk<T, D>& walk) {
    const int64_t seen = (int64_t)walk.seq.base + p.by_group.quotient((uint32_t)walk.block.first) + 1;
    return (int32_t)(max((int64_t)0, min(seen, (int64_t)walk.block.end)) / CaShape<D>::KT);
}

// Three warps copy token by token: pages of fewer than eight tokens, or of an odd number.
template <typename T, int D>
__device__ __noinline__ void ca_load(const CaParams<T>& p, CaControl<D>* ctl, char* queries, char* stages) {
    using S = CaShape<D>;
    CaLoader<T, D> load;
    load.ctl = ctl;
    load.bars = ca_smem(ctl);
    load.stages = ca_smem(stages);
    const uint32_t q_at = ca_smem(queries);
    const int32_t t = (int32_t)threadIdx.x - 256, warp = t / 32;
    CaWalk<T, D> walk(p, ctl->place[0], ctl->bound[0], ctl->bound[1]);
    uint32_t q_phase = 1, meeting = 0;
    int32_t tiles_done = 0;
    while (walk.next()) {
        const auto& b = walk.block;
        const int32_t* table = p.tables + walk.seq_number * p.table_stride;
        auto page_of = [&](int32_t token) -> int32_t {
            if (token >= b.end) return -1;
            const int32_t page = table[p.by_page.quotient((uint32_t)token)];
            return page >= 0 && page < p.pages ? page : -1;
        };
        if (walk.tile1 == walk.tile0) continue;                          // no token to see
        // (the tile's tokens to the threads, the last 32 of 128 to the first warp once more)
        int32_t page = t < S::KT ? page_of(walk.tile0 * S::KT + t) : -1, page2 = t + CA_LOADERS < S::KT ? page_of(walk.tile0 * S::KT + CA_LOADERS + t) : -1;
        if (!load.wait(CA_AT(load.bars, q_free), q_phase)) break;
        q_phase ^= 1;
        // (the scores of the item before are made: so all warps are through with the item CA_ITEMS before this one, whose bits these were)
        if (t < CA_BAD_TILES * 4) ctl->bad[walk.number % CA_ITEMS][t / 4][t % 4] = 0;
        if (t == 0) ctl->any_bad[walk.number % CA_ITEMS] = 0;
        ca_copy_queries<T, D>(p, walk, q_at, t, CA_LOAD_ROWS);
        load.issued(CA_AT(load.bars, q_full), -1);
        const int32_t cut = ca_first_cut<T, D>(p, walk);
        const T* keys = p.k + walk.head * p.ks_head;
        const T* values = p.v + walk.head * p.vs_head;
        bool ok = true;
        for (int32_t tile = walk.tile0; tile < walk.tile1 && ok; ++tile, ++tiles_done) {
            const int32_t buffer = tiles_done & 1;
            const uint32_t there = __ballot_sync(FULL_MASK, page >= 0), there2 = __ballot_sync(FULL_MASK, page2 >= 0);
            uint32_t* mask = ctl->mask[tiles_done % CA_MASKS];
            if (t < S::KT) ctl->table[buffer][t] = page;
            if (t + CA_LOADERS < S::KT) ctl->table[buffer][t + CA_LOADERS] = page2;
            if (lane_id() == 0) {
                mask[warp] = warp * 32 < S::KT ? there : ~0u;
                if (warp == 0) mask[3] = CA_LOADERS < S::KT ? there2 : ~0u;
            }
            if (tile + 1 < walk.tile1) {
                page = t < S::KT ? page_of((tile + 1) * S::KT + t) : -1;
                page2 = t + CA_LOADERS < S::KT ? page_of((tile + 1) * S::KT + CA_LOADERS + t) : -1;
            }
            if (!(ok = ca_meet(CA_AT(load.bars, loaders), meeting, ctl->failed))) break;
            const int32_t first = tile * S::KT;
            ok = load.tile(p, keys, p.ks_page, p.ks_token, buffer, first, -1);
            ok = ok && load.tile(p, values, p.vs_page, p.vs_token, buffer, first, tile >= cut ? (tile % CA_BAD_TILES) << 8 | (walk.number % CA_ITEMS) << 16 : -1);
        }
        if (!ok) break;
    }
    load.flush();
    asm volatile("cp.async.wait_all;" ::: "memory");
}

__device__ __forceinline__ void ca_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ca_tile_copy(uint32_t to, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y, int32_t z, int32_t w) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(to), "l"(map), "r"(bar), "r"(x),
                 "r"(y), "r"(z), "r"(w)
                 : "memory");
}

// One warp has tiles copied in boxes of 64 elements and up to a tile's tokens of a page, a lane to each.  A page that is not
// there lies outside the described memory: the copy fills in zeros.
template <typename T, int D>
__device__ void ca_load_boxes(const CaParams<T>& p, const CaMaps& maps, CaControl<D>* ctl, uint32_t queries, uint32_t stages) {
    using S = CaShape<D>;
    const int32_t lane = (int32_t)lane_id(), boxes = S::KT / p.box, box = lane % boxes, half = lane / boxes;
    const uint32_t to = (uint32_t)(half * S::KT * 128 + box * p.box * 128), bars = ca_smem(ctl);
    CaWalk<T, D> walk(p, ctl->place[0], ctl->bound[0], ctl->bound[1]);
    uint32_t q_phase = 1, phase = 1;
    int32_t stage = 0, tiles_done = 0;
    bool ok = true;
    while (ok && walk.next()) {
        const auto& b = walk.block;
        if (walk.tile1 == walk.tile0) continue;                          // no token to see
        const int32_t* table = p.tables + walk.seq_number * p.table_stride;
        int32_t slot = 0, next_slot = 0;
        auto page_of = [&](int32_t token, int32_t* at) -> int32_t {
            if (token >= b.end) return p.pages;
            const uint32_t c = p.by_page.quotient((uint32_t)token);
            *at = token - (int32_t)(c * p.by_page.d);
            const int32_t page = table[c];
            return page >= 0 && page < p.pages ? page : p.pages;
        };
        int32_t next = page_of(walk.tile0 * S::KT + box * p.box, &next_slot);
        if (p.q_box) {
            const int32_t streams = b.rows > CA_ROWS ? 2 : 1;
            if (!(ok = ca_wait(CA_AT(bars, q_free), q_phase, ctl->failed))) break;
            q_phase ^= 1;
            if (lane == 0) ca_expect(CA_AT(bars, q_full), streams * S::Q_TILE);
            __syncwarp();
            if (lane < streams * (D / 64)) {
                const int32_t s = lane / (D / 64), h = lane % (D / 64), token = (int32_t)p.by_group.quotient((uint32_t)(b.first + s * CA_ROWS));
                ca_tile_copy(queries + s * S::Q_TILE + h * CA_ROWS * 128, &maps.q, CA_AT(bars, q_full), h * 64, walk.head * p.group, (p.starts ? walk.seq.row0 : 0) + token,
                             p.starts ? 0 : walk.seq_number);
            }
        }
        for (int32_t tile = walk.tile0; ok && tile < walk.tile1; ++tile, ++tiles_done) {
            const int32_t page = next;
            slot = next_slot;
            const uint32_t there = __ballot_sync(FULL_MASK, page < p.pages);
            if (lane < 4) {                                              // a box's bit to its tokens' bits
                uint32_t word = 0;
                for (int32_t i = 0; i < 32; i += 8) word |= (there >> (uint32_t)min((lane * 32 + i) / p.box, 31) & 1u) * 0xFFu << i;
                ctl->mask[tiles_done % CA_MASKS][lane] = lane * 32 < S::KT ? word : ~0u;
            }
            if (tile + 1 < walk.tile1) next = page_of((tile + 1) * S::KT + box * p.box, &next_slot);
            __syncwarp();
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                if (!(ok = ca_wait(CA_AT(bars, empty) + stage * 8, phase, ctl->failed))) break;
                if (lane == 0) ca_expect(CA_AT(bars, full) + stage * 8, S::STAGE);
                __syncwarp();
                if (half < D / 64) ca_tile_copy(stages + stage * S::STAGE + to, kv ? &maps.v : &maps.k, CA_AT(bars, full) + stage * 8, half * 64, slot, walk.head, page);
                if (++stage == S::STAGES) { stage = 0; phase ^= 1; }
            }
        }
    }
    // Nothing may land behind the CTA's end: should a wait have run out somewhere, nobody else waits for these copies.  (A phase
    // of a barrier that has had none is over.)
    if (p.q_box) ca_drain(CA_AT(bars, q_full), q_phase);
    for (int32_t st = 0; st < S::STAGES; ++st) ca_drain(CA_AT(bars, full) + st * 8, st < stage ? phase ^ 1u : phase);
}

// Two warps beside it look through the tiles of values that a mask cuts before they are multiplied, and copy the queries where
// that cannot be done by tile.
template <typename T, int D>
__device__ void ca_look(const CaParams<T>& p, CaControl<D>* ctl, uint32_t queries, uint32_t stages) {
    using S = CaShape<D>;
    const int32_t t = (int32_t)threadIdx.x - 256 - 32;
    const uint32_t bars = ca_smem(ctl);
    CaWalk<T, D> walk(p, ctl->place[0], ctl->bound[0], ctl->bound[1]);
    uint32_t q_phase = p.q_box ? 0 : 1, meeting = 0, asked = 0;
    int32_t taken = 0;
    while (walk.next()) {
        const int32_t n = walk.tile1 - walk.tile0;
        if (n == 0) continue;
        if (!ca_wait(p.q_box ? CA_AT(bars, q_full) : CA_AT(bars, q_free), q_phase, ctl->failed)) break;
        q_phase ^= 1;
        if (!p.q_box) {
            ca_copy_queries<T, D>(p, walk, queries, t, 64 / 8);
            asm volatile("cp.async.wait_all;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane_id() == 0) ca_arrive(CA_AT(bars, q_full));
        }
        if (t < CA_BAD_TILES * 4) ctl->bad[walk.number % CA_ITEMS][t / 4][t % 4] = 0;
        if (t == 0) ctl->any_bad[walk.number % CA_ITEMS] = 0;
        // (products of an item begin behind this, so these warps are never an item ahead)
        if (!ca_meet(CA_AT(bars, opened), meeting, ctl->failed)) break;
        bool ok = true;
        for (int32_t tile = max(walk.tile0, ca_first_cut<T, D>(p, walk)); tile < walk.tile1 && ok; ++tile) {
            const int32_t number = taken + 2 * (tile - walk.tile0) + 1, st = number % S::STAGES;
            // asked for once the stage's use before this one has passed: then its parity is this one's
            ok = ca_wait(CA_AT(bars, asked), asked, ctl->failed) && ca_wait(CA_AT(bars, full) + st * 8, (uint32_t)(number / S::STAGES) & 1u, ctl->failed);
            asked ^= 1;
            if (!ok) break;
            CaLoader<T, D>::template look<64 / 8>(ctl, stages, st, tile % CA_BAD_TILES, walk.number % CA_ITEMS, t);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane_id() == 0) ca_arrive(CA_AT(bars, looked));
        }
        if (!ok) break;
        taken += 2 * n;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// ---- products ----------------------------------------------------------------------------------

// A place in the ring of stages: every second one, keys or values.
template <int D>
struct CaCursor {
    using S = CaShape<D>;
    uint32_t bars, stages;                // shared memory: the control block, the stages
    uint32_t stage, parity = 0;
    __device__ __forceinline__ uint32_t full() const { return CA_AT(bars, full) + stage * 8; }
    __device__ __forceinline__ uint32_t empty() const { return CA_AT(bars, empty) + stage * 8; }
    __device__ __forceinline__ uint32_t data() const { return stages + stage * S::STAGE; }
    __device__ __forceinline__ void step() {
        stage += 2;
        if (stage >= S::STAGES) { stage -= S::STAGES; parity ^= 1u; }
    }
};

// One warp issues all products of the CTA: all its lanes wait and walk, one is elected to issue.
template <typename T, int D>
__device__ void ca_multiply(const CaParams<T>& p, CaControl<D>* ctl, uint32_t queries, uint32_t stages) {
    using S = CaShape<D>;
    const uint32_t tm = ca_uniform(ctl->tensor), bars = ca_smem(ctl);
    const uint32_t one = ca_elect();
    constexpr uint32_t SCORES = ca_product<T>(S::KT, false), OUTPUT = ca_product<T>(D, true);
    CaWalk<T, D> walk(p, ctl->place[0], ctl->bound[0], ctl->bound[1]);
    uint32_t q_phase = 0, p_phases = 0, opened = 0, look_phase = 0;      // p_phases: a bit for each place of scores
    CaCursor<D> k{bars, stages, 0}, v{bars, stages, 1};
    auto wait = [&](uint32_t bar, uint32_t parity) { return ca_wait(bar, parity, ctl->failed); };
    auto weights = [&](int buffer) {
        const bool ok = wait(CA_AT(bars, p_full) + buffer * 8, p_phases >> buffer & 1u);
        p_phases ^= 1u << buffer;
        ca_after_sync();
        return ok;
    };
    // S = Q K^T, and whom it concerns
    auto scores = [&](int s, int buffer) {
        const uint32_t q = ca_uniform(ca_operand_low(queries + s * S::Q_TILE, 16)), k0 = ca_uniform(ca_operand_low(k.data(), 16)), to = ca_uniform(tm + buffer * 128);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            ca_mma_ss(to, ca_operand(q + i / 4 * (CA_ROWS * 8) + i % 4 * 2), ca_operand(k0 + i / 4 * (S::KT * 8) + i % 4 * 2), SCORES, i > 0, one);
        ca_commit(CA_AT(bars, s_full) + buffer * 8, one);
    };
    // O += P V
    auto output = [&](int o, int buffer, bool add) {
        const uint32_t v0 = ca_uniform(ca_operand_low(v.data(), S::KT * 128)), to = ca_uniform(tm + S::O_AT + o * D), from = ca_uniform(tm + buffer * 128);
        ca_mma_ts(to, from, ca_operand(v0), OUTPUT, add, one);
#pragma unroll
        for (int i = 1; i < S::KT / 16; ++i) ca_mma_ts(to, from + i * 8, ca_operand(v0 + i * 128), OUTPUT, true, one);
    };
    bool some = walk.next();
    while (some) {
        const int32_t n = walk.tile1 - walk.tile0;
        if (n == 0) {
            some = walk.next();
            continue;
        }
        if (!wait(CA_AT(bars, q_full), q_phase)) return;
        q_phase ^= 1u;
        // Values that a mask cuts are looked through first: by those that copied them, or by warps that tell of it.  One tile is
        // asked for at a time: the first when the keys of the tile before it are here, the next ones in turn.
        const int32_t cut = p.box ? max(ca_first_cut<T, D>(p, walk) - walk.tile0, 0) : n, ask = cut < n ? max(cut - 1, 0) : -1;
        auto keys = [&](int32_t i) {
            if (!wait(k.full(), k.parity)) return false;
            if (i == ask && one) ca_arrive(CA_AT(bars, asked));
            ca_after_sync();
            return true;
        };
        auto values = [&](int32_t i) {
            if (!wait(v.full(), v.parity)) return false;
            if (i < cut) return true;
            const bool ok = wait(CA_AT(bars, looked), look_phase);
            look_phase ^= 1u;
            if (one && i + 1 < n) ca_arrive(CA_AT(bars, asked));
            return ok;
        };
        if (p.box) {
            if (!wait(CA_AT(bars, opened), opened)) return;
            opened ^= 1u;
        }
        if (!keys(0)) return;
        const bool both = S::STREAMS == 2 && walk.block.rows > CA_ROWS;
        scores(0, 0);
        if (both) scores(1, 1);
        ca_commit(k.empty(), one);
        if (n == 1) ca_commit(CA_AT(bars, q_free), one);
        k.step();
        if (both) {
            // both streams over every tile
#pragma unroll 1
            for (int32_t i = 0; i < n; ++i) {
                if (!values(i)) return;
                if (i + 1 == n) some = walk.next();                      // (while the last weights are made)
#pragma unroll 1
                for (int st = 0; st < 2; ++st) {
                    if (!weights(st)) return;
                    output(st, st, i > 0);
                    if (i + 1 < n) {
                        if (st == 0 && !keys(i + 1)) return;
                        scores(st, st);
                    } else {
                        ca_commit(CA_AT(bars, o_full) + st * 8, one);
                    }
                }
                // (told of last: a commit between the products of a stream and its next scores delays those)
                ca_commit(v.empty(), one);
                if (i + 1 < n) ca_commit(k.empty(), one);
                if (i + 2 == n) ca_commit(CA_AT(bars, q_free), one);
                v.step();
                if (i + 1 < n) k.step();
            }
        } else {
            // tiles alternate between two places of scores (and, with two streams, two of output)
#pragma unroll 1
            for (int32_t i = 0; i < n; ++i) {
                const int buffer = i & 1;
                if (i + 1 < n) {
                    if (!keys(i + 1)) return;
                    scores(0, buffer ^ 1);
                    ca_commit(k.empty(), one);
                    if (i + 2 == n) ca_commit(CA_AT(bars, q_free), one);
                    k.step();
                }
                if (!values(i)) return;
                if (i + 1 == n) some = walk.next();
                if (!weights(buffer)) return;
                output(S::STREAMS == 2 ? buffer : 0, buffer, i >= S::STREAMS);
                ca_commit(v.empty(), one);
                if constexpr (S::STREAMS == 2) {
                    if (i + 2 >= n) ca_commit(CA_AT(bars, o_full) + buffer * 8, one);
                } else {
                    ca_commit(CA_AT(bars, o_step), one);
                    if (i + 1 == n) ca_commit(CA_AT(bars, o_full), one);
                }
                v.step();
            }
        }
    }
}

// ---- weights and output ------------------------------------------------------------------------

struct CaWho { int32_t seq, head, row0, tile0, tile1; };                 // an item's

// Adds what tokens with values that are not finite contribute to 32 columns of a row's output (their values were left out of
// the product, where they would have met weights of zero).  Slow, and rare: the token's weight is computed again.
template <typename T, int D>
__device__ __noinline__ void ca_add_bad(const CaParams<T>& p, const uint32_t (*bad)[4], const CaWho& who, uint32_t row_token, uint32_t g, int32_t seen, float factor,
                                        float reference, int32_t column, float* o) {
    using S = CaShape<D>;
    const int32_t* table = p.tables + who.seq * p.table_stride;
    const T* q = p.q + (p.starts ? (int64_t)who.row0 * p.q_token : who.seq * p.q_seq) + row_token * p.q_token + ((int64_t)who.head * p.group + g) * p.q_head;
    for (int32_t tile = max(who.tile0, who.tile1 - CA_BAD_TILES); tile < who.tile1; ++tile)
        for (int32_t i = 0; i < S::KT; ++i) {
            const int64_t token = (int64_t)tile * S::KT + i;
            if (!(bad[tile % CA_BAD_TILES][i / 32] >> (i % 32) & 1u) || token >= seen) continue;
            const int64_t page = table[token / p.page_size], slot = token % p.page_size;
            const T* k = p.k + page * p.ks_page + who.head * p.ks_head + slot * p.ks_token;
            const T* v = p.v + page * p.vs_page + who.head * p.vs_head + slot * p.vs_token;
            float s = 0.0f;
            for (int32_t d = 0; d < p.dim; ++d) s += Logit<T>::to_float(q[d]) * Logit<T>::to_float(k[d]);
            const float w = exp2_approx(s * factor - reference);
            // in vectors of 16 bytes, as they were taken out
            for (int32_t c = 0; c < 32 && column + c < p.dim; c += 8) {
                bool out = false;
                for (int e = 0; e < 8; ++e) out |= !isfinite(Logit<T>::to_float(v[column + c + e]));
                for (int e = 0; out && e < 8; ++e) o[c + e] += w * Logit<T>::to_float(v[column + c + e]);
            }
        }
}

// A warpgroup's part: a thread to a row.
template <typename T, int D>
__device__ void ca_weigh(const CaParams<T>& p, CaControl<D>* ctl) {
    using S = CaShape<D>;
    constexpr int KT = S::KT;
    const int group = (int)threadIdx.x / 128, lane_row = (int)threadIdx.x % 128;          // (stream, row of its tile)
    const uint32_t lanes = (uint32_t)(lane_row / 32) << 21;                               // this warp's lanes of the tensor memory
    const uint32_t tm = ctl->tensor + lanes;
    volatile int32_t* failed = ctl->failed;
    const float factor = p.scale * LOG2E;
    CaWalk<T, D> walk(p, ctl->place[0], ctl->bound[0], ctl->bound[1]);
    const uint32_t bars = ca_smem(ctl);
    uint32_t s_phases = 0, o_phase = 0, step_phase = 0, meeting = 0;     // s_phases: a bit for each place of scores
    int32_t tiles_done = 0;
    bool more = walk.next();
    while (more) {
        const auto b = walk.block;
        const bool both = S::STREAMS == 2 && b.rows > CA_ROWS;           // streams have rows of their own
        const int32_t n = walk.tile1 - walk.tile0;
        const int32_t row = (both ? group * CA_ROWS : 0) + lane_row;     // of the item
        const bool held = row < b.rows, warp_held = (row & ~31) < b.rows;
        const uint32_t token = p.by_group.quotient((uint32_t)(b.first + min(row, b.rows - 1))), g = (uint32_t)(b.first + min(row, b.rows - 1)) - token * p.group;
        const int32_t seen = (int32_t)max(-1ll, min((long long)walk.seq.base + token + 1, (long long)b.end));       // tokens of the row
        const int32_t first = both || S::STREAMS == 1 ? 0 : group, step = both || S::STREAMS == 1 ? 1 : 2;
        float reference = LOWEST, sum = 0.0f, lost = 0.0f;
        bool ok = true;
        for (int32_t i = first; i < n; i += step) {
            const int buffer = both ? group : (S::STREAMS == 2 ? group : i & 1);
            ok = ca_wait(CA_AT(bars, s_full) + buffer * 8, s_phases >> buffer & 1u, failed);
            if (!ok) break;
            s_phases ^= 1u << buffer;
            ca_after_sync();
            if (warp_held) {
                float x[KT];
#pragma unroll
                for (int c = 0; c < KT; c += 32) ca_tm_load(tm + buffer * 128 + c, x + c);
#pragma unroll
                for (int c = 0; c < KT; c += 32) ca_tm_loaded(x + c);
                const uint4 mask = *reinterpret_cast<const uint4*>(ctl->mask[(tiles_done + i) % CA_MASKS]);
                const int32_t left = seen - (walk.tile0 + i) * KT;
                if (left < KT || (mask.x & mask.y & mask.z & mask.w) != ~0u) {
                    const uint32_t word[4] = {mask.x, mask.y, mask.z, mask.w};
#pragma unroll
                    for (int c0 = 0; c0 < KT; c0 += 32) {
                        const int32_t there = left - c0;                 // tokens of this word that the row sees
                        const uint32_t on = word[c0 / 32] & (there >= 32 ? ~0u : there <= 0 ? 0u : (1u << there) - 1u);
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (!(on & 1u << c)) x[c0 + c] = -INFINITY;
                    }
                }
                float most[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                for (int c = 4; c < KT; ++c) most[c % 4] = fmaxf(most[c % 4], x[c]);
                const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * factor;
                const bool raise = top > reference + CaType<T>::RAISE;
                if (__any_sync(FULL_MASK, raise)) {
                    const float next = raise ? top : reference, by = raise ? exp2_approx(reference - next) : 1.0f;
                    reference = next;
                    sum *= by;
                    lost *= by;
                    if (i > first) {
                        if (S::STREAMS == 1) {           // the products of the tile before may still run
                            ok = ca_wait(CA_AT(bars, o_step), step_phase ^ 1u, failed);
                            ca_after_sync();
                        }
                        const uint32_t o = tm + S::O_AT + (S::STREAMS == 2 ? group * D : 0);
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            float y[32];
                            ca_tm_load(o + c, y);
                            ca_tm_loaded(y);
#pragma unroll
                            for (int e = 0; e < 32; ++e) y[e] *= by;
                            ca_tm_store(o + c, reinterpret_cast<uint32_t*>(y));
                        }
                    }
                }
                const F32x2 by = f2_make(factor, factor), minus = f2_make(CaType<T>::LIFT - reference, CaType<T>::LIFT - reference);
                F32x2 part[4];
#pragma unroll
                for (int c0 = 0; c0 < KT; c0 += 32) {
                    uint32_t packed[16];
#pragma unroll
                    for (int c = c0; c < c0 + 32; c += 2) {
                        float u, v;
                        f2_split(f2_fma(f2_make(x[c], x[c + 1]), by, minus), u, v);
                        u = exp2_approx(u);
                        v = exp2_approx(v);
                        const F32x2 w = f2_make(u, v);
                        part[c / 2 % 4] = c < 8 ? w : f2_add(part[c / 2 % 4], w);
                        packed[(c - c0) / 2] = CaType<T>::pack(u, v);
                    }
                    ca_tm_store16(tm + buffer * 128 + c0 / 2, packed);
                }
                float u, v;
                f2_split(f2_add(f2_add(part[0], part[1]), f2_add(part[2], part[3])), u, v);
                const float y = (u + v) - lost, more = sum + y;          // (what a sum loses is taken off the next addend)
                lost = (more - sum) - y;
                sum = more;
                ca_tm_stored();
            }
            step_phase ^= 1;
            ca_before_sync();
            __syncwarp();
            if (lane_id() == 0) ca_arrive(CA_AT(bars, p_full) + buffer * 8);
            if (!ok) break;
        }
        if (!ok) break;
        // --- the item's output: this thread's row.  (The next item is found while the last products run.)
        const int32_t tile0 = walk.tile0, number = walk.number;
        const bool whole = walk.whole();
        const CaWho who{walk.seq_number, walk.head, walk.seq.row0, tile0, walk.tile1};
        more = walk.next();
        const bool shared = S::STREAMS == 2 && !both;                    // two streams share rows: the first writes
        const bool mine = both || group == 0;
        const int32_t others = shared ? n / 2 : 0;                       // tiles of the second stream
        if (n > first) {
            ok = ca_wait(CA_AT(bars, o_full) + (S::STREAMS == 2 ? group * 8 : 0), o_phase, failed);
            if (!ok) break;
            o_phase ^= 1;
        }
        float lift = 1.0f, other_lift = 0.0f;
        if (shared && n > 0) {
            if (group == 1) ctl->other[lane_row] = make_float2(reference, sum);
            ca_before_sync();
            if (!ca_meet(CA_AT(bars, weighers), meeting, failed)) break;
            ca_after_sync();
            if (mine && others > 0) {
                const float2 o = ctl->other[lane_row];
                const float most = fmaxf(reference, o.x);
                lift = exp2_approx(reference - most);
                other_lift = exp2_approx(o.x - most);
                sum = sum * lift + o.y * other_lift;
                reference = most;
            }
        }
        ca_after_sync();
        if (mine && warp_held) {
            const int64_t out_row = (int64_t)(who.row0 + token) * p.heads + (int64_t)who.head * p.group + g;
            const int32_t slot = (int32_t)blockIdx.x * 2 + (tile0 == 0 ? 1 : 0);
            float* part = whole ? nullptr : p.parts + ((int64_t)slot * S::BLOCK + row) * D;
            // (of a sum of zero, all products are zeros, too)
            const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
            const bool any_bad = n > 0 && ctl->any_bad[number % CA_ITEMS] != 0;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                if (c >= p.dim) break;
                __syncwarp();
                float y[32];
                if (n > 0) {
                    ca_tm_load(tm + S::O_AT + (both ? group * D : 0) + c, y);
                    ca_tm_loaded(y);
                    if (others > 0) {
                        float z[32];
                        ca_tm_load(tm + S::O_AT + D + c, z);
                        ca_tm_loaded(z);
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = y[e] * lift + z[e] * other_lift;
                    }
                    if (any_bad && held) {
                        float z[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) z[e] = y[e];
                        ca_add_bad<T, D>(p, ctl->bad[number % CA_ITEMS], who, token, g, seen, factor, reference - CaType<T>::LIFT, c, z);
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = z[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[e] = 0.0f;
                }
                if (!held) continue;
                if (part) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(part + c + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        if (c + e >= p.dim) break;
                        float f[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = y[e + j] * inverse;
                        *reinterpret_cast<uint4*>(p.out + out_row * p.dim + c + e) = Logit<T>::pack(f);
                    }
                }
            }
            if (held) {
                if (whole) p.lse[out_row] = sum == 0.0f ? -INFINITY : (reference - CaType<T>::LIFT + log2f(sum)) * 0.6931471805599453f;
                else p.sums[(int64_t)slot * S::BLOCK + row] = make_float2(reference, sum);
            }
            if (!whole && row == 0) {
                CaMeta* m = p.meta + slot;
                m->valid = 1;
                m->last = who.tile1 == b.tiles;
                m->rows = b.rows;
                m->row0 = who.row0;
                m->head = who.head;
                m->first = b.first;
            }
        }
        ca_before_sync();
        if (shared && n > 0 && !ca_meet(CA_AT(bars, weighers), meeting, failed)) break;
        ca_after_sync();
        tiles_done += n;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(CA_THREADS, 1) paged_attention_chunk_kernel(const __grid_constant__ CaParams<T> p, const __grid_constant__ CaMaps maps) {
    using S = CaShape<D>;
    extern __shared__ __align__(1024) char ca_memory[];
    char* queries = ca_memory;
    char* stages = ca_memory + S::STREAMS * S::Q_TILE;
    CaControl<D>* ctl = reinterpret_cast<CaControl<D>*>(stages + S::STAGES * S::STAGE);
    const uint32_t bars = ca_smem(ctl);
    const int32_t warp = (int32_t)threadIdx.x / 32;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) {
            ca_bar_init(CA_AT(bars, full) + i * 8, p.box ? 1 : CA_LOADERS / 32);
            ca_bar_init(CA_AT(bars, empty) + i * 8, 1);
        }
        ca_bar_init(CA_AT(bars, q_full), !p.box ? CA_LOADERS / 32 : p.q_box ? 1 : 2);
        ca_bar_init(CA_AT(bars, opened), 2);
        ca_bar_init(CA_AT(bars, asked), 1);
        ca_bar_init(CA_AT(bars, looked), 2);
        ca_bar_init(CA_AT(bars, q_free), 1);
        for (int i = 0; i < 2; ++i) {
            ca_bar_init(CA_AT(bars, s_full) + i * 8, 1);
            ca_bar_init(CA_AT(bars, p_full) + i * 8, 4);
            ca_bar_init(CA_AT(bars, o_full) + i * 8, 1);
        }
        ca_bar_init(CA_AT(bars, o_step), 1);
        ca_bar_init(CA_AT(bars, loaders), CA_LOADERS / 32);
        ca_bar_init(CA_AT(bars, weighers), 8);
        ca_bar_init(CA_AT(bars, drain), 1);
        ctl->failed[0] = 0;
        ctl->failed[1] = p.polls;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 11) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(ca_smem(&ctl->tensor)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        ca_before_sync();
    }
    pdl_wait();
    pdl_launch_dependents();
    if (threadIdx.x < 2) {
        CaMeta* m = p.meta + blockIdx.x * 2 + threadIdx.x;
        m->valid = m->last = m->failed = 0;
    }
    ca_plan<T, D>(p, ctl);
    ca_after_sync();
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(CA_MANY_REGISTERS));
        if (p.starts) {
            // rows that no sequence holds
            const int64_t a = max(0, min(p.starts[0], p.rows)), z = max(a, (int64_t)min(p.starts[p.seqs], p.rows));
            const int64_t t = (int64_t)blockIdx.x * 256 + (int)threadIdx.x, all = (int64_t)gridDim.x * 256;
            const int64_t per = (int64_t)p.heads * p.dim / 8, n = a + p.rows - z;
            for (int64_t i = t; i < n * per; i += all) {
                const int64_t r = i / per, row = r < a ? r : r - a + z;
                reinterpret_cast<uint4*>(p.out)[row * per + i % per] = make_uint4(0, 0, 0, 0);
            }
            for (int64_t i = t; i < n * p.heads; i += all) {
                const int64_t r = i / p.heads, row = r < a ? r : r - a + z;
                p.lse[row * p.heads + i % p.heads] = -INFINITY;
            }
            __syncwarp();
        }
        if (S::STREAMS == 2 || warp < 4) ca_weigh<T, D>(p, ctl);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(CA_FEW_REGISTERS));
        if (warp < 11) {
            if (!p.box) ca_load<T, D>(p, ctl, queries, stages);
            else if (warp == 8) ca_load_boxes<T, D>(p, maps, ctl, ca_smem(queries), ca_smem(stages));
            else ca_look<T, D>(p, ctl, ca_smem(queries), ca_smem(stages));
        } else {
            ca_multiply<T, D>(p, ctl, ca_smem(queries), ca_smem(stages));
        }
    }
    ca_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && ctl->failed[0]) p.meta[blockIdx.x * 2].failed = 1;
    if (warp == 11) {
        if (ctl->failed[0]) {                                            // products may be under way still: those of the lane that issues them
            ca_commit(CA_AT(bars, drain), ca_elect());
            ca_drain(CA_AT(bars, drain), 0);
        }
        ca_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(ctl->tensor));
    }
}

// Joins the parts of the item that begins in CTA x's share and goes on in the next ones'; rows are spread over grid.y.
constexpr int CJ_THREADS = 256;
template <typename T, int D>
__global__ void __launch_bounds__(CJ_THREADS) paged_attention_chunk_join_kernel(const CaParams<T> p, int32_t ctas) {
    using S = CaShape<D>;
    pdl_wait();
    pdl_launch_dependents();
    // (a wait of the first kernel that ran out leaves its outputs unwritten: then none are given)
    bool failed = false;
    for (int32_t c = (int32_t)threadIdx.x; c < ctas; c += CJ_THREADS) failed |= p.meta[c * 2].failed != 0;
    if (__syncthreads_or(failed)) {
        const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * CJ_THREADS + threadIdx.x, all = (int64_t)gridDim.x * gridDim.y * CJ_THREADS;
        for (int64_t i = t; i < (int64_t)p.rows * p.heads * p.dim; i += all) p.out[i] = Logit<T>::from_float(NAN);
        for (int64_t i = t; i < (int64_t)p.rows * p.heads; i += all) p.lse[i] = NAN;
        return;
    }
    const int32_t c0 = (int32_t)blockIdx.x;
    const CaMeta m = p.meta[c0 * 2 + 1];
    if (!m.valid) return;
    const int32_t warp = (int32_t)threadIdx.x / 32, lane = (int32_t)lane_id();
    int32_t last = c0 + 1;                                               // the CTA with the item's last part
    for (uint32_t found = 0; last < ctas; last += 32) {
        found = __ballot_sync(FULL_MASK, last + lane < ctas && p.meta[(last + lane) * 2].last != 0);
        if (found) { last += __ffs((int)found) - 1; break; }
    }
    last = min(last, ctas - 1);
    auto slot_of = [&](int32_t c) { return (int64_t)(c == c0 ? c0 * 2 + 1 : c * 2); };
    for (int32_t row = (int32_t)blockIdx.y * (CJ_THREADS / 32) + warp; row < m.rows; row += (int32_t)gridDim.y * (CJ_THREADS / 32)) {
        float most = LOWEST;
        for (int32_t c = c0 + lane; c <= last; c += 32) most = fmaxf(most, p.sums[slot_of(c) * S::BLOCK + row].x);
        for (int d = 16; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(FULL_MASK, most, d));
        float sum = 0.0f, o[D / 32] = {};
#pragma unroll 4
        for (int32_t c = c0; c <= last; ++c) {
            const float2 s = p.sums[slot_of(c) * S::BLOCK + row];
            const float by = exp2_approx(s.x - most);
            sum += s.y * by;
            const float* part = p.parts + (slot_of(c) * S::BLOCK + row) * D;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) o[j] += part[lane + 32 * j] * by;
        }
        const uint32_t r = (uint32_t)(m.first + row), token = p.by_group.quotient(r), g = r - token * p.group;
        const int64_t out_row = (int64_t)(m.row0 + token) * p.heads + (int64_t)m.head * p.group + g;
        const float inverse = 1.0f / sum;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            if (lane + 32 * j < p.dim) p.out[out_row * p.dim + lane + 32 * j] = Logit<T>::from_float(sum == 0.0f ? 0.0f : o[j] * inverse);
        }
        if (lane == 0) p.lse[out_row] = sum == 0.0f ? -INFINITY : (most - CaType<T>::LIFT + log2f(sum)) * 0.6931471805599453f;
    }
}

}  // namespace profk
