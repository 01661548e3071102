// Pages of a key-value cache that sequences share: forking, growing, releasing, compacting, copying, appending.
//
// A sequence is a row of a page table and a length; refs[p] counts the table entries that hold page p, 0 means free.
// What a call decides (who keeps a page, which free page goes where) is settled by one small kernel with prefix sums, in
// an order that the definition gives, so that the result does not depend on timing; a second kernel over the whole
// device then writes tables and counts and moves the pages' bytes.
#pragma once

#include "common.cuh"

namespace profk {

constexpr int PG_PLAN_THREADS = 1024;
constexpr int PG_THREADS = 256;
// 16-byte vectors per thread in flight, and CTAs per SM.  Whole pages: fewer CTAs with more in flight each (1 GB moved: 171 us
// against 179); the shorter pieces that a fork copies: more CTAs (86 MB: 24 us against 28).
constexpr int PG_UNROLL_PAGES = 8, PG_CTAS_PAGES = 4;
constexpr int PG_UNROLL_PIECES = 4, PG_CTAS_PIECES = 6;

// Where a pool's bytes lie; strides in bytes, all multiples of 16.
struct PgPool {
    char* base;                           // null: no pool, tables and counts only
    int32_t layers, kv_heads, page_size;
    int32_t row_bytes;                    // of one token and head
    int32_t team;                         // threads that copy one plane of a page (a power of two, 32 .. PG_THREADS)
    int64_t layer, kv, page, head, token;
};

struct PgMove { int32_t src, dst, tokens, unused; };

struct PgPlanHead {                       // first words of the workspace
    int32_t moves;                        // pages to copy
    int32_t live;                         // compaction: live pages
    int32_t fresh;                        // fork: free pages found
    int32_t unused;
};

struct PgForkParams {
    const int32_t* tables;
    int64_t table_stride;
    const int32_t* lengths;
    const int32_t* refs;
    const int32_t* parents;
    int32_t n_old, n, width, pages, page_size, grow;
    bool past_room;                       // lengths go on behind the table's end
    int32_t* out_tables;                  // n x width
    int32_t* out_lengths;
    int32_t* out_refs;
    int32_t* out_missing;
    PgPlanHead* head;
    int32_t* first;                       // n_old: lowest child, or n
    int32_t* kids;                        // n_old
    int32_t* need;                        // n: number of the sequence's first fresh page
    int32_t* fresh;                       // lowest free pages, ascending
    PgMove* moves;                        // n
    PgPool pool;
};

__device__ __forceinline__ int32_t pg_length(const int32_t* lengths, int32_t s, int32_t width, int32_t page_size) {
    const int64_t room = (int64_t)width * page_size;
    return (int32_t)max((int64_t)0, min((int64_t)lengths[s], room));
}
__device__ __forceinline__ int32_t pg_ceil(int64_t tokens, int32_t page_size) { return (int32_t)((tokens + page_size - 1) / page_size); }

constexpr int PG_NEAR = 4096;             // old sequences whose children are counted in shared memory

struct PgChild {
    int32_t parent, old, length, counted, have, want, fill, beyond;   // parent < 0: an empty sequence; beyond: pages past the table
    bool copy;
    __device__ __forceinline__ PgChild(const PgForkParams& p, int32_t i) : PgChild(p, i, p.first) {}
    __device__ __forceinline__ PgChild(const PgForkParams& p, int32_t i, const int32_t* first) {
        parent = p.parents[i];
        if (parent < 0 || parent >= p.n_old) parent = -1;
        old = parent >= 0 ? pg_length(p.lengths, parent, p.width, p.page_size) : 0;
        const int64_t wanted = (int64_t)old + p.grow;
        length = (int32_t)min(wanted, (int64_t)p.width * p.page_size);
        counted = p.past_room ? (int32_t)min(wanted, (int64_t)0x7FFFFFFF) : length;
        have = pg_ceil(old, p.page_size);
        want = pg_ceil(length, p.page_size);
        beyond = pg_ceil(wanted, p.page_size) - want;
        fill = old % p.page_size;
        copy = parent >= 0 && fill > 0 && first[parent] != i;
    }
    __device__ __forceinline__ int32_t fresh_from() const { return have - (copy ? 1 : 0); }   // columns from here on are fresh
};

// Block-wide sum of the numbers before this thread's, and of all of them (1024 threads).
__device__ __forceinline__ uint32_t pg_scan(uint32_t v, uint32_t* warp_sums, uint32_t* total) {
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5;
    uint32_t incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t up = __shfl_up_sync(FULL_MASK, incl, d);
        if (lane >= (uint32_t)d) incl += up;
    }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    const uint32_t w = warp_sums[lane];                  // (32 warps)
    *total = __reduce_add_sync(FULL_MASK, w);
    const uint32_t before = __reduce_add_sync(FULL_MASK, lane < warp ? w : 0u);
    __syncthreads();                                     // warp_sums may be used again
    return before + incl - v;
}

// Block 0 plans; the others copy the counts, which the second kernel then changes.
__global__ void __launch_bounds__(PG_PLAN_THREADS) pages_fork_plan_kernel(const PgForkParams p) {
    __shared__ uint32_t warp_sums[32];
    __shared__ int32_t s_moves;
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x > 0) {
        for (int64_t i = (int64_t)(blockIdx.x - 1) * PG_PLAN_THREADS + tid; i < p.pages; i += (int64_t)(gridDim.x - 1) * PG_PLAN_THREADS)
            p.out_refs[i] = p.refs[i];
        return;
    }
    __shared__ int32_t s_first[PG_NEAR], s_kids[PG_NEAR];
    const bool near = p.n_old <= PG_NEAR;
    int32_t* first = near ? s_first : p.first;
    int32_t* kids = near ? s_kids : p.kids;
    if (tid == 0) s_moves = 0;
    for (int32_t s = tid; s < p.n_old; s += PG_PLAN_THREADS) { first[s] = p.n; kids[s] = 0; }
    __syncthreads();
    for (int32_t i = tid; i < p.n; i += PG_PLAN_THREADS) {
        const int32_t parent = p.parents[i];
        if (parent >= 0 && parent < p.n_old) {
            atomicMin(&first[parent], i);
            atomicAdd(&kids[parent], 1);
        }
    }
    __syncthreads();
    if (near)
        for (int32_t s = tid; s < p.n_old; s += PG_PLAN_THREADS) { p.first[s] = first[s]; p.kids[s] = kids[s]; }
    // how many fresh pages each new sequence needs, numbered through
    uint32_t total = 0, beyond = 0;
    for (int32_t i0 = 0; i0 < p.n; i0 += PG_PLAN_THREADS) {
        const int32_t i = i0 + tid;
        uint32_t mine = 0, sum = 0;
        if (i < p.n) {
            const PgChild c(p, i, first);
            mine = (uint32_t)(c.want - c.fresh_from());
            beyond += (uint32_t)c.beyond;
            p.out_lengths[i] = c.counted;
        }
        const uint32_t before = pg_scan(mine, warp_sums, &sum);
        if (i < p.n) p.need[i] = (int32_t)(total + before);
        total += sum;
    }
    // the lowest-numbered free pages, a walk by this CTA that ends with the last one needed (256 sequences: 15 us where the free
    // pages lie low, 34 where they are the last of 100,000, 210 the last of a million)
    uint32_t found = 0;
    for (int32_t c0 = 0; c0 < p.pages && found < total; c0 += 4 * PG_PLAN_THREADS) {
        const int32_t at = c0 + 4 * tid;
        bool is_free[4];
        uint32_t mine = 0, sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            is_free[j] = at + j < p.pages && p.refs[at + j] <= 0;
            mine += is_free[j];
        }
        uint32_t number = found + pg_scan(mine, warp_sums, &sum);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (is_free[j]) {
                if (number < total) p.fresh[number] = at + j;
                ++number;
            }
        found += sum;
    }
    found = min(found, total);
    __syncthreads();
    // the partly filled pages that are copied
    for (int32_t i = tid; i < p.n; i += PG_PLAN_THREADS) {
        const PgChild c(p, i, first);
        if (!c.copy) continue;
        const int32_t src = p.tables[c.parent * p.table_stride + c.have - 1], number = p.need[i];
        if (number < (int32_t)found && src >= 0 && src < p.pages) {
            const int32_t slot = atomicAdd(&s_moves, 1);                       // (their order is of no consequence)
            p.moves[slot] = PgMove{src, p.fresh[number], c.fill, 0};
        }
    }
    uint32_t all_beyond;
    pg_scan(beyond, warp_sums, &all_beyond);
    if (tid == 0) {
        *p.head = PgPlanHead{s_moves, 0, (int32_t)found, 0};
        *p.out_missing = (int32_t)(total - found + all_beyond);
    }
}

// One page of one layer's keys or values: `tokens` tokens of every head, by `pool.team` threads.  A whole CTA for each would
// idle on small ones (20,000 planes of 1.5 KB, 32 MB: 73 us with the plan, a warp for each 28; 160,000 of 4 KB: 310 us, 115).
template <int PG_UNROLL>
__device__ __forceinline__ void pg_copy(const PgPool& pool, int32_t src, int32_t dst, int32_t tokens, int32_t plane) {
    const uint32_t team = (uint32_t)pool.team, rank = threadIdx.x & (team - 1);
    char* base = pool.base + (plane >> 1) * pool.layer + (plane & 1) * pool.kv;
    const char* from = base + src * pool.page;
    char* to = base + dst * pool.page;
    // runs of bytes that lie together: all tokens of a head, all heads of a token, or neither
    int64_t run_stride = pool.token, outer_stride = pool.head;
    uint32_t run = (uint32_t)pool.row_bytes / 16, runs = (uint32_t)tokens, outer = (uint32_t)pool.kv_heads;
    if (pool.token == pool.row_bytes) {
        run *= (uint32_t)tokens;
        runs = 1;
    } else if (pool.head == pool.row_bytes) {
        run *= (uint32_t)pool.kv_heads;
        outer = 1;
    }
    const uint32_t n = run * runs * outer;
    auto offset = [&](uint32_t i) {
        const uint32_t r = i / run, o = r / runs;
        return (int64_t)o * outer_stride + (int64_t)(r - o * runs) * run_stride + (int64_t)(i - r * run) * 16;
    };
    for (uint32_t i0 = rank; i0 < n; i0 += team * PG_UNROLL) {
        uint4 x[PG_UNROLL];
        int64_t at[PG_UNROLL];
#pragma unroll
        for (int u = 0; u < PG_UNROLL; ++u) {
            const uint32_t i = i0 + u * team;
            if (i < n) {
                at[u] = offset(i);
                x[u] = *reinterpret_cast<const uint4*>(from + at[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < PG_UNROLL; ++u)
            if (i0 + u * team < n) *reinterpret_cast<uint4*>(to + at[u]) = x[u];
    }
}

// The thread's team among all teams of the grid, and their number.
__device__ __forceinline__ int64_t pg_team(const PgPool& pool) { return ((int64_t)blockIdx.x * PG_THREADS + threadIdx.x) / pool.team; }
__device__ __forceinline__ int64_t pg_teams(const PgPool& pool) { return (int64_t)gridDim.x * (PG_THREADS / pool.team); }

// The copies of a plan; no page is both read and written by them.
template <int PG_UNROLL>
__device__ __forceinline__ void pg_copy_all(const PgPool& pool, const PgMove* moves, int32_t n) {
    if (!pool.base) return;
    const int32_t planes = 2 * pool.layers;
    for (int64_t unit = pg_team(pool); unit < (int64_t)n * planes; unit += pg_teams(pool)) {
        const PgMove m = moves[unit / planes];
        pg_copy<PG_UNROLL>(pool, m.src, m.dst, m.tokens, (int32_t)(unit % planes));
    }
}

__global__ void __launch_bounds__(PG_THREADS) pages_fork_kernel(const PgForkParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const PgPlanHead head = *p.head;
    const int64_t step = (int64_t)gridDim.x * PG_THREADS, me = (int64_t)blockIdx.x * PG_THREADS + threadIdx.x;
    for (int64_t e = me; e < (int64_t)p.n * p.width; e += step) {
        const int32_t i = (int32_t)(e / p.width), col = (int32_t)(e % p.width);
        const PgChild c(p, i);
        int32_t page = -1;
        if (col < c.want) {
            if (col < c.fresh_from()) {
                page = p.tables[c.parent * p.table_stride + col];
                if (page < 0 || page >= p.pages) page = -1;
            } else {
                const int32_t number = p.need[i] + col - c.fresh_from();
                if (number < head.fresh) {
                    page = p.fresh[number];
                    atomicAdd(&p.out_refs[page], 1);
                }
            }
        }
        p.out_tables[e] = page;
    }
    // An old sequence held each of its pages once; its children hold the full ones once each, the first of them the
    // partly filled one too.
    for (int64_t e = me; e < (int64_t)p.n_old * p.width; e += step) {
        const int32_t s = (int32_t)(e / p.width), col = (int32_t)(e % p.width);
        const int32_t len = pg_length(p.lengths, s, p.width, p.page_size), kids = p.kids[s];
        if (col >= pg_ceil(len, p.page_size)) continue;
        const bool partial = col == len / p.page_size;
        const int32_t change = (partial ? min(kids, 1) : kids) - 1;
        if (change == 0) continue;
        const int32_t page = p.tables[s * p.table_stride + col];
        if (page >= 0 && page < p.pages) atomicAdd(&p.out_refs[page], change);
    }
    pg_copy_all<PG_UNROLL_PIECES>(p.pool, p.moves, head.moves);
}

// ---- compaction ------------------------------------------------------------------------------

constexpr int32_t PG_FREE = -1, PG_STAYS = -2;

struct PgCompactParams {
    const int32_t* tables;
    int64_t table_stride;
    const int32_t* refs;
    int32_t n, width, pages;
    int32_t* out_tables;                  // n x width
    int32_t* out_refs;
    int32_t* page_map;
    int32_t* out_live;
    PgPlanHead* head;
    int32_t* to;                          // pages: PG_FREE, PG_STAYS, or the number of the move that takes the page
    int32_t share;                        // pages that a planning CTA settles
    PgMove* moves;                        // pages / 2
    PgPool pool;
};

// Live pages among [from, to), block-wide.
__device__ __forceinline__ uint32_t pg_live(const int32_t* refs, int64_t from, int64_t to, uint32_t* warp_sums) {
    uint32_t mine = 0, sum = 0;
#pragma unroll 8
    for (int64_t i = from + threadIdx.x; i < to; i += PG_PLAN_THREADS) mine += refs[i] > 0;
    pg_scan(mine, warp_sums, &sum);
    return sum;
}

// Live pages behind the first `live` go to the free ones among them, both in ascending order.  Every CTA settles a share of
// the pages and counts for itself what lies before it: reading all counts again (4 bytes per page, from L2) costs less than a
// walk by one CTA with a prefix sum per step (100,000 pages, half of them free,
// with the copies: 52 us, with the walk 140), and nothing waits for another CTA.
__global__ void __launch_bounds__(PG_PLAN_THREADS) pages_compact_plan_kernel(const PgCompactParams p) {
    __shared__ uint32_t warp_sums[32];
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    const int64_t from = (int64_t)blockIdx.x * p.share, to = min((int64_t)p.pages, from + p.share);
    const uint32_t before = pg_live(p.refs, 0, from, warp_sums);
    const uint32_t live = before + pg_live(p.refs, from, p.pages, warp_sums);
    uint32_t holes = from <= live ? (uint32_t)from - before : 0;               // (behind `live` there are none to number)
    uint32_t movers = from > live ? pg_live(p.refs, live, from, warp_sums) : 0;
    for (int64_t c0 = from; c0 < to; c0 += 4 * PG_PLAN_THREADS) {
        const int64_t at = c0 + 4 * tid;
        uint32_t n_holes = 0, n_movers = 0, sum_holes = 0, sum_movers = 0;
        int32_t ref[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ref[j] = at + j < to ? p.refs[at + j] : 0;
            const bool held = ref[j] > 0, low = at + j < live;
            n_holes += low && !held && at + j < to;
            n_movers += !low && held;
        }
        uint32_t hole = holes + pg_scan(n_holes, warp_sums, &sum_holes), mover = movers + pg_scan(n_movers, warp_sums, &sum_movers);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (at + j >= to) break;
            const int32_t page = (int32_t)(at + j);
            const bool held = ref[j] > 0, low = at + j < live;
            p.out_refs[page] = low && held ? ref[j] : 0;
            p.page_map[page] = low && held ? page : -1;
            p.to[page] = !held ? PG_FREE : low ? PG_STAYS : (int32_t)mover;
            if (low && !held) p.moves[hole++].dst = page;
            if (!low && held) {
                p.moves[mover].src = page;
                p.moves[mover++].tokens = p.pool.page_size;
            }
        }
        holes += sum_holes;
        movers += sum_movers;
    }
    if (tid == 0 && to == p.pages) {
        // as many movers as holes: the live pages that do not lie among the first `live`
        *p.head = PgPlanHead{(int32_t)movers, (int32_t)live, 0, 0};
        *p.out_live = (int32_t)live;
    }
}

__global__ void __launch_bounds__(PG_THREADS) pages_compact_kernel(const PgCompactParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int32_t moves = p.head->moves;
    const int64_t step = (int64_t)gridDim.x * PG_THREADS, me = (int64_t)blockIdx.x * PG_THREADS + threadIdx.x;
    for (int64_t i = me; i < moves; i += step) {
        const PgMove m = p.moves[i];
        p.page_map[m.src] = m.dst;
        p.out_refs[m.dst] = p.refs[m.src];
    }
    for (int64_t e = me; e < (int64_t)p.n * p.width; e += step) {
        const int32_t page = p.tables[e / p.width * p.table_stride + e % p.width];
        const int32_t to = page >= 0 && page < p.pages ? p.to[page] : PG_FREE;
        p.out_tables[e] = to >= 0 ? p.moves[to].dst : to == PG_STAYS ? page : -1;
    }
    pg_copy_all<PG_UNROLL_PAGES>(p.pool, p.moves, moves);
}

// ---- copying given pages, appending tokens -----------------------------------------------------

struct PgCopyParams {
    const int32_t* src;
    const int32_t* dst;
    int32_t n, pages;
    PgPool pool;
};

__global__ void __launch_bounds__(PG_THREADS) pages_copy_kernel(const PgCopyParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int32_t planes = 2 * p.pool.layers;
    for (int64_t unit = pg_team(p.pool); unit < (int64_t)p.n * planes; unit += pg_teams(p.pool)) {
        const int32_t src = p.src[unit / planes], dst = p.dst[unit / planes];
        if (src < 0 || src >= p.pages || dst < 0 || dst >= p.pages || src == dst) continue;
        pg_copy<PG_UNROLL_PAGES>(p.pool, src, dst, p.pool.page_size, (int32_t)(unit % planes));
    }
}

// Keys and values of the last `tokens` tokens of every sequence go to their places.  Lengths are taken as they are: the tokens
// of a sequence that has outgrown its table have none (taken into the table, they would overwrite its last tokens, in pages that
// other sequences may hold).
struct PgAppendParams {
    const char* k;                        // seqs x tokens x kv_heads rows; strides in bytes
    const char* v;
    int64_t k_seq, k_tok, k_head, v_seq, v_tok, v_head;
    char* k_pages;
    char* v_pages;
    int64_t kp_page, kp_head, kp_token, vp_page, vp_head, vp_token;
    const int32_t* tables;
    int64_t table_stride;
    const int32_t* lengths;
    int32_t seqs, tokens, kv_heads, row_bytes, page_size, pages, width;
};

__global__ void __launch_bounds__(PG_THREADS) pages_append_kernel(const PgAppendParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int32_t vecs = p.row_bytes / 16;
    const int64_t n = (int64_t)p.seqs * p.tokens * p.kv_heads * vecs;
    for (int64_t i = (int64_t)blockIdx.x * PG_THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * PG_THREADS) {
        const int32_t vec = (int32_t)(i % vecs);
        int64_t rest = i / vecs;
        const int32_t head = (int32_t)(rest % p.kv_heads);
        rest /= p.kv_heads;
        const int32_t tok = (int32_t)(rest % p.tokens), seq = (int32_t)(rest / p.tokens);
        const int64_t place = (int64_t)p.lengths[seq] - p.tokens + tok;
        if (place < 0 || place >= (int64_t)p.width * p.page_size) continue;
        const int32_t at = (int32_t)place;
        const int32_t page = p.tables[seq * p.table_stride + at / p.page_size], slot = at % p.page_size;
        if (page < 0 || page >= p.pages) continue;
        const uint4 k = *reinterpret_cast<const uint4*>(p.k + seq * p.k_seq + tok * p.k_tok + head * p.k_head + vec * 16);
        const uint4 v = *reinterpret_cast<const uint4*>(p.v + seq * p.v_seq + tok * p.v_tok + head * p.v_head + vec * 16);
        *reinterpret_cast<uint4*>(p.k_pages + page * p.kp_page + head * p.kp_head + slot * p.kp_token + vec * 16) = k;
        *reinterpret_cast<uint4*>(p.v_pages + page * p.vp_page + head * p.vp_head + slot * p.vp_token + vec * 16) = v;
    }
}

}  // namespace profk
