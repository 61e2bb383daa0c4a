// Pages of the pool: which rows hold which blocks.  Rows are handed on (fork), grow (extend), are freed (release,
// trim), and blocks in use are moved to the lowest ids (compact); tables and counts live in device memory.
//
// Bound: latency.  The bytes are few (a table of 128 rows of 8192 ids is 4 MB, counts of a million blocks 4 MB, all in L2), each
// kernel is a launch and three to six rounds of loads that depend on each other.  On a B200, in a captured graph: fork of 64 rows
// of 160 entries 4.7 us, of 128 rows of 8200 7.8; extend of 64 rows 5.0-6.4, of 1024 rows among a million blocks 7.4; trim of 64 rows of
// 1040 entries 1.9, of 1024 of 520 3.7; release 1.7; compact of 5000 blocks 6.0.
// Two things grow with the call: an extension's new blocks are given out by one CTA, 1.1 us a thousand (by 512 blocks 5.5 us, 4096 9.4,
// 32768 43, 524288 597), and the rows are seen by every CTA of fork, or by one of extend (65536 rows: fork 500 us, extend 219, trim 42).
#include <new>

#include "tutti_attend.h"

namespace tutti {

namespace {

constexpr uint32_t PLAN_THREADS = 1024;
constexpr uint32_t TILE = 4 * PLAN_THREADS;     // counts that a CTA looks at in one round
constexpr uint32_t ROW_THREADS = 256;
constexpr uint32_t ROW_IDS = 8 * ROW_THREADS;   // ids of a row that a CTA takes at once
constexpr uint32_t GROUP = 16;                  // old rows whose counts a CTA of fork changes together
constexpr uint32_t SEARCH = 4096;               // rows whose first ranks fit in shared memory
constexpr uint32_t SMALL = 16;                  // tiles that every CTA of a compaction counts by itself

struct TablesDev {
    uint32_t n_seq, n_blk, block_tokens;
    const uint32_t *blk_start;
    int32_t *block_ids;
    uint32_t *len;
    int32_t *status;
};

// The handle's memory.  arrive, turn, writers and top are zero between calls.
struct PagesDev {
    int32_t *refs;
    uint32_t n_blocks, n_tiles;
    uint32_t *arrive;                           // CTAs of extend that are done
    uint32_t *turn;                             // [max rows] CTAs of release that have read a row's length
    uint32_t *tile;                             // [n_tiles] free blocks, or blocks in use
    uint32_t *moves;                            // of a compaction
    unsigned long long *total;                  // new blocks of an extension
    uint32_t *writers, *top;                    // [n_blocks] rows that write to a shared block, and the last of them + 1
    uint32_t *rank;                             // [n_blocks] a moved block's number; free blocks of extend, from each tile's start on
    uint32_t *begin, *entry;                    // [max rows] rank of a row's first new block, and where it goes
    int32_t *mark, *keep_id, *keep_count;       // [max rows] see plan_rows
};

__device__ inline void report(int32_t *status, int code) {
    if (status) atomicCAS(status, TUTTI_OK, code);
}

struct Row {
    uint32_t b0, room, len, held;
};

__host__ __device__ inline uint32_t blocks_of(uint32_t tokens, uint32_t block_tokens) {
    return tokens / block_tokens + (tokens % block_tokens != 0);
}

// The entries of row s, without its length.
__device__ inline bool row_room(const TablesDev &t, uint32_t s, Row &r) {
    const uint32_t b0 = t.blk_start[s], b1 = t.blk_start[s + 1];
    if (b0 > b1 || b1 > t.n_blk) return false;
    r.b0 = b0;
    r.room = b1 - b0;
    return true;
}
__device__ inline bool row_view(const TablesDev &t, uint32_t s, Row &r) {
    r.len = t.len[s];
    if (!row_room(t, s, r) || r.len > 0x7fffffffu) return false;
    r.held = blocks_of(r.len, t.block_tokens);
    return r.held <= r.room;
}

// One holder less; a count that is 0 stays 0.
__device__ inline void drop(const PagesDev &p, int32_t id, int32_t *status) {
    if (atomicAdd(p.refs + id, -1) <= 0) {
        atomicAdd(p.refs + id, 1);
        report(status, TUTTI_EINVAL);
    }
}

// What goes back to a count that `sum` has taken to `now`: as much of `sum` as lies below 0.  (Not all that lies below 0: several
// may take from one count at once, and each gives back its own part.)
__host__ __device__ inline int given_back(int now, int sum) { return now >= 0 || sum >= 0 ? 0 : now > sum ? -now : -sum; }

// Sum over the CTA's threads before this one; `total` over all.  sums: [32] in shared memory.
template <typename U>
__device__ inline U scan(U x, U *sums, U &total) {
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31, warps = blockDim.x / 32;
    U incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const U y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    __syncthreads();                            // the sums of an earlier scan have been read
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    U w = lane < warps ? sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const U y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const U before = __shfl_sync(0xffffffffu, w, warp ? warp - 1 : 0);
    return incl - x + (warp ? before : 0);
}

// The four counts of a thread in a tile; blocks behind the last one read as `none`.
__device__ inline int4 tile_counts(const PagesDev &p, uint32_t tile, int none) {
    const uint32_t id = tile * TILE + threadIdx.x * 4;
    if (id + 4 <= p.n_blocks) return *reinterpret_cast<const int4 *>(p.refs + id);
    int4 v = make_int4(none, none, none, none);
    if (id < p.n_blocks) v.x = p.refs[id];
    if (id + 1 < p.n_blocks) v.y = p.refs[id + 1];
    if (id + 2 < p.n_blocks) v.z = p.refs[id + 2];
    return v;
}
__device__ inline uint32_t zeros(const int4 &v) { return (v.x == 0) + (v.y == 0) + (v.z == 0) + (v.w == 0); }

// ---------------------------------------------------------------------------------------------
// fork: CTAs [0, per * to.n_seq) copy the entries of the new rows, the ones behind change the counts of the old
// rows' blocks, by as many as a row has children (less the row itself, where it is given up).  A CTA takes GROUP
// old rows together and adds up what neighbours that hold the same block at the same place do to its count: the beams of
// a request share their prompt, and what one loses there another gains, so that most blocks need no atomic at all.
__global__ void __launch_bounds__(ROW_THREADS) fork_kernel(const PagesDev p, const TablesDev from, const int32_t *parent, const TablesDev to, uint32_t move, uint32_t per, uint32_t segs) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t row = blockIdx.x / per, part = blockIdx.x % per;
    Row r, child;
    if (row < to.n_seq) {
        const int32_t f = parent[row];
        bool ok = row_room(to, row, child);
        if (f != -1) ok = ok && (uint32_t)f < from.n_seq && row_view(from, f, r) && r.held <= child.room;
        if (part == 0 && threadIdx.x == 0) {
            to.len[row] = ok && f != -1 ? r.len : 0;
            if (!ok) report(to.status, TUTTI_EINVAL);
        }
        if (!ok || f == -1) return;
        const int32_t *src = from.block_ids + r.b0;
        int32_t *dst = to.block_ids + child.b0;
        for (uint32_t i0 = part * ROW_IDS; i0 < r.held; i0 += per * ROW_IDS) {
            int32_t id[ROW_IDS / ROW_THREADS];
#pragma unroll
            for (uint32_t k = 0; k < ROW_IDS / ROW_THREADS; ++k) {
                const uint32_t i = i0 + k * ROW_THREADS + threadIdx.x;
                if (i < r.held) id[k] = src[i];
            }
#pragma unroll
            for (uint32_t k = 0; k < ROW_IDS / ROW_THREADS; ++k) {
                const uint32_t i = i0 + k * ROW_THREADS + threadIdx.x;
                if (i < r.held) dst[i] = id[k];
            }
        }
        return;
    }
    __shared__ uint32_t first[GROUP], held[GROUP], longest;
    __shared__ int by[GROUP];
    const uint32_t g = blockIdx.x - per * to.n_seq, f0 = g % ((from.n_seq + GROUP - 1) / GROUP) * GROUP, seg = g / ((from.n_seq + GROUP - 1) / GROUP);
    if (threadIdx.x == 0) longest = 0;
    // the thread's first child, and its room, are fetched along with the old rows
    int32_t parent0 = -1;
    bool room0 = false;
    Row child0;
    child0.room = 0;
    if (threadIdx.x < to.n_seq) {
        parent0 = parent[threadIdx.x];
        room0 = row_room(to, threadIdx.x, child0);
    }
    __syncthreads();
    if (threadIdx.x < GROUP) {
        const uint32_t f = f0 + threadIdx.x;
        const bool there = f < from.n_seq, ok = there && row_view(from, f, r);
        if (there && !ok && seg == 0) report(from.status, TUTTI_EINVAL);
        first[threadIdx.x] = ok ? r.b0 : 0;
        held[threadIdx.x] = ok ? r.held : 0;
        by[threadIdx.x] = move ? -1 : 0;
        if (ok) atomicMax(&longest, r.held);
    }
    __syncthreads();
    if (seg * ROW_THREADS >= longest) return;
    for (uint32_t c = threadIdx.x; c < to.n_seq; c += ROW_THREADS) {
        const bool is_first = c == threadIdx.x;
        const uint32_t k = (uint32_t)(is_first ? parent0 : parent[c]) - f0;
        if (k >= GROUP || !(is_first ? room0 : row_room(to, c, child))) continue;
        if (held[k] <= (is_first ? child0.room : child.room)) atomicAdd(by + k, 1);
    }
    __syncthreads();
    for (uint32_t i = seg * ROW_THREADS + threadIdx.x; i < longest; i += segs * ROW_THREADS) {
        int32_t id[GROUP];
#pragma unroll
        for (uint32_t k = 0; k < GROUP; ++k) id[k] = i < held[k] ? from.block_ids[first[k] + i] : -1;
        int32_t run = -1;
        int sum = 0;
        auto flush = [&]() {
            if (run == -1 || (sum == 0 && !move)) return;       // (nobody takes it, and it is kept)
            if ((uint32_t)run >= p.n_blocks) {
                report(from.status, TUTTI_EFAULT);
                return;
            }
            if (sum == 0) return;
            const int now = atomicAdd(p.refs + run, sum) + sum;
            if (now < 0) {                      // a count does not pass 0
                if (const int back = given_back(now, sum)) atomicAdd(p.refs + run, back);
                report(from.status, TUTTI_EINVAL);
            }
        };
#pragma unroll
        for (uint32_t k = 0; k < GROUP; ++k) {
            if (id[k] != run) {
                flush();
                run = id[k];
                sum = 0;
            }
            sum += by[k];
        }
        flush();
    }
}

// ---------------------------------------------------------------------------------------------
// extend: CTA 0 decides which rows copy and ranks the new blocks of all rows by a prefix sum, the others count the free
// blocks of a tile each and list them; the last to arrive gives block number k to its row.
struct Growth {
    Row r;
    uint32_t add, more;
    int32_t tail;                               // the partly filled block that is written to, or -1
    int32_t count;                              // its count
    int code;
};
__device__ inline Growth growth(const PagesDev &p, const TablesDev &t, const uint32_t *n_new, uint32_t s) {
    Growth g;
    g.add = n_new[s];
    g.tail = -1;
    g.count = 1;
    g.more = 0;
    g.code = TUTTI_EINVAL;
    if (!row_view(t, s, g.r) || g.add > 0x7fffffffu - g.r.len) return g;
    const uint32_t after = blocks_of(g.r.len + g.add, t.block_tokens);
    if (after > g.r.room) return g;
    if (g.add && g.r.len % t.block_tokens) {
        const int32_t id = t.block_ids[g.r.b0 + g.r.len / t.block_tokens];
        if (id != -1) {
            if ((uint32_t)id >= p.n_blocks) {
                g.code = TUTTI_EFAULT;
                return g;
            }
            g.count = p.refs[id];
            if (g.count <= 0) return g;
            g.tail = id;
        }
    }
    g.more = after - g.r.held;
    g.code = TUTTI_OK;
    return g;
}

// mark: the block that a row copies, -1 none, -2 the row is skipped.  keep_id, keep_count: what a shared block's
// count becomes, at the last of its writers.
__device__ void plan_rows(const PagesDev &p, const TablesDev &t, const uint32_t *n_new, unsigned long long *sums) {
    Growth own;                                 // the thread's last row (its only one, mostly)
    uint32_t own_s = ~0u;
    auto look = [&](uint32_t s) {
        if (s != own_s) own = growth(p, t, n_new, s);
        own_s = s;
    };
    // Rows that write to a block that others hold: how many, and which is the last.
    bool shares = false;
    for (uint32_t s = threadIdx.x; s < t.n_seq; s += PLAN_THREADS) {
        look(s);
        if (own.code != TUTTI_OK) report(t.status, own.code);
        else if (own.count > 1) {
            atomicAdd(p.writers + own.tail, 1);
            atomicMax(p.top + own.tail, s + 1);
            shares = true;
        }
    }
    shares = __syncthreads_or(shares);
    unsigned long long total = 0;
    for (uint32_t s0 = 0; s0 < t.n_seq; s0 += PLAN_THREADS) {
        const uint32_t s = s0 + threadIdx.x;
        bool copies = false, ok = false;
        if (s < t.n_seq) {
            look(s);
            ok = own.code == TUTTI_OK;
            int32_t keep = -1;
            if (shares && ok && own.count > 1) {
                const int32_t w = (int32_t)__ldcg(p.writers + own.tail);
                const bool is_last = __ldcg(p.top + own.tail) == s + 1;
                copies = !(is_last && w >= own.count);
                if (is_last) {
                    keep = own.tail;
                    p.keep_count[s] = w < own.count ? own.count - w : 1;
                }
            }
            p.keep_id[s] = keep;
            p.mark[s] = !ok ? -2 : copies ? own.tail : -1;
        }
        unsigned long long all;
        const unsigned long long before = scan<unsigned long long>(ok ? own.more + copies : 0, sums, all);
        if (s < t.n_seq) {
            p.begin[s] = (uint32_t)(total + before);
            p.entry[s] = ok ? own.r.b0 + own.r.held - copies : 0;
        }
        total += all;
    }
    if (threadIdx.x == 0) *p.total = total;
}

// The last of `begin`'s rows (ascending, begin[0] = 0) that starts at k or before.
__device__ inline uint32_t last_at(const uint32_t *begin, uint32_t n, uint32_t k) {
    uint32_t lo = 0;
    while (n > 1) {
        const uint32_t half = n / 2;
        if (begin[lo + half] <= k) lo += half, n -= half;
        else n = half;
    }
    return lo;
}

__global__ void __launch_bounds__(PLAN_THREADS) extend_kernel(const PagesDev p, const TablesDev t, const uint32_t *n_new, int32_t *pairs) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ unsigned long long sums[32];
    __shared__ uint32_t sums32[32], first[PLAN_THREADS], ranks[SEARCH], entries[PLAN_THREADS];
    __shared__ bool last, copies[PLAN_THREADS];
    if (blockIdx.x == 0) {
        plan_rows(p, t, n_new, sums);
    } else {
        const uint32_t tile = blockIdx.x - 1, id = tile * TILE + threadIdx.x * 4;
        const int4 v = tile_counts(p, tile, 1);
        uint32_t n, k = scan(zeros(v), sums32, n);
        // as many as all rows together may need
        uint32_t *list = p.rank + (uint64_t)tile * TILE;
        if (v.x == 0 && k < t.n_blk) list[k] = id;
        k += v.x == 0;
        if (v.y == 0 && k < t.n_blk) list[k] = id + 1;
        k += v.y == 0;
        if (v.z == 0 && k < t.n_blk) list[k] = id + 2;
        k += v.z == 0;
        if (v.w == 0 && k < t.n_blk) list[k] = id + 3;
        if (threadIdx.x == 0) p.tile[tile] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        last = arrive_gpu(p.arrive) == gridDim.x - 1;
        if (last) *p.arrive = 0;                // ready for the next call
    }
    __syncthreads();
    if (!last) return;

    // Everything that the end needs is fetched in one go: the thread's row and tile are its only ones, mostly.
    const unsigned long long total = __ldcg(p.total);
    const uint32_t me = threadIdx.x;
    int32_t keep = -1, mark = -2, keep_count = 0;
    uint32_t begin = 0, len = 0, add = 0, entry = 0, mine = 0;
    auto fetch = [&](uint32_t s) {
        keep = __ldcg(p.keep_id + s), mark = __ldcg(p.mark + s), keep_count = __ldcg(p.keep_count + s);
        begin = __ldcg(p.begin + s), entry = __ldcg(p.entry + s), len = t.len[s], add = n_new[s];
    };
    if (me < t.n_seq) fetch(me);
    const uint32_t c0 = me < p.n_tiles ? __ldcg(p.tile + me) : 0;
    for (uint32_t i = me + PLAN_THREADS; i < p.n_tiles; i += PLAN_THREADS) mine += __ldcg(p.tile + i);
    uint32_t in_first, n_free;                  // in the first tiles, and in all
    const uint32_t before0 = scan(c0, sums32, in_first);
    n_free = in_first;
    if (p.n_tiles > PLAN_THREADS) {
        scan(mine, sums32, n_free);
        n_free += in_first;
    }
    // more new blocks than entries: rows that lie over each other
    const bool enough = total <= n_free && total <= t.n_blk;
    if (!enough && me == 0) report(t.status, total <= t.n_blk ? TUTTI_EAGAIN : TUTTI_EINVAL);
    // The rows' new lengths and counts of the blocks that they shared.
    for (uint32_t s = me; s < t.n_seq; s += PLAN_THREADS) {
        if (s != me) fetch(s);
        if (s < SEARCH) ranks[s] = begin;
        if (s < PLAN_THREADS) entries[s] = entry, copies[s] = mark >= 0;
        if (keep >= 0) p.writers[keep] = p.top[keep] = 0;
        if (keep >= 0 && enough) p.refs[keep] = keep_count;
        if (mark != -2 && enough) t.len[s] = len + add;
        pairs[2 * s] = enough && mark >= 0 ? mark : -1;
        if (!enough || mark < 0) pairs[2 * s + 1] = -1;
    }
    if (!enough) return;
    uint32_t at = 0;                            // free blocks in front of the tiles in hand
    for (uint32_t t0 = 0; t0 < p.n_tiles && at < total; t0 += PLAN_THREADS) {
        uint32_t in_all = in_first;
        if (t0 == 0) {
            first[me] = before0;
        } else {
            const uint32_t c = t0 + me < p.n_tiles ? __ldcg(p.tile + t0 + me) : 0;
            first[me] = at + scan(c, sums32, in_all);
        }
        __syncthreads();
        for (uint32_t k = at + threadIdx.x; k < total && k < at + in_all; k += PLAN_THREADS) {
            const uint32_t i = last_at(first, PLAN_THREADS, k);
            const uint32_t id = __ldcg(p.rank + (uint64_t)(t0 + i) * TILE + (k - first[i]));
            const uint32_t s = t.n_seq <= SEARCH ? last_at(ranks, t.n_seq, k) : last_at(p.begin, t.n_seq, k);
            const uint32_t j = k - (t.n_seq <= SEARCH ? ranks[s] : p.begin[s]);
            const bool here = s < PLAN_THREADS;
            t.block_ids[(here ? entries[s] : __ldcg(p.entry + s)) + j] = (int32_t)id;
            if (j == 0 && (here ? copies[s] : __ldcg(p.mark + s) >= 0)) pairs[2 * s + 1] = (int32_t)id;
            p.refs[id] = 1;
        }
        at += in_all;
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------
// release and trim: `per` CTAs a row.  Release clears a row's length once all its CTAs have read it: the last to
// say so does it, and the entries are independent of that.
__global__ void __launch_bounds__(ROW_THREADS) release_kernel(const PagesDev p, const TablesDev t, const uint8_t *which, uint32_t per) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t s = blockIdx.x / per, part = blockIdx.x % per;
    if (which && !which[s]) return;
    Row r;
    const bool ok = row_view(t, s, r);
    __syncthreads();
    if (threadIdx.x == 0) {
        if (!ok && part == 0) report(t.status, TUTTI_EINVAL);
        if (ok && (per == 1 || arrive_gpu(p.turn + s) == per - 1)) {
            if (per > 1) p.turn[s] = 0;
            t.len[s] = 0;
        }
    }
    if (!ok) return;
    for (uint32_t i = part * ROW_THREADS + threadIdx.x; i < r.held; i += per * ROW_THREADS) {
        const int32_t id = t.block_ids[r.b0 + i];
        if (id == -1) continue;
        t.block_ids[r.b0 + i] = -1;
        if ((uint32_t)id >= p.n_blocks) report(t.status, TUTTI_EFAULT);
        else drop(p, id, t.status);
    }
}

__global__ void __launch_bounds__(ROW_THREADS) trim_kernel(const PagesDev p, const TablesDev t, uint32_t window, uint32_t sinks, uint32_t per) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t s = blockIdx.x / per, part = blockIdx.x % per;
    Row r;
    if (!row_view(t, s, r)) {
        if (part == 0 && threadIdx.x == 0) report(t.status, TUTTI_EINVAL);
        return;
    }
    if (r.len < window) return;
    const uint32_t end = (r.len - window + 1) / t.block_tokens;
    for (uint32_t i = blocks_of(sinks, t.block_tokens) + part * ROW_THREADS + threadIdx.x; i < end; i += per * ROW_THREADS) {
        const int32_t id = t.block_ids[r.b0 + i];
        if (id == -1) continue;
        t.block_ids[r.b0 + i] = -1;
        if ((uint32_t)id >= p.n_blocks) report(t.status, TUTTI_EFAULT);
        else drop(p, id, t.status);
    }
}

// ---------------------------------------------------------------------------------------------
// compact, with u(i) the blocks in use below i and n all of them: a free block f < n is the destination
// number f - u(f), a block in use s >= n is the source number n - 1 - u(s), and there are n - u(n) of each.
__global__ void __launch_bounds__(PLAN_THREADS) compact_count_kernel(const PagesDev p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ uint32_t sums[32];
    uint32_t n;
    scan(4 - zeros(tile_counts(p, blockIdx.x, 0)), sums, n);
    if (threadIdx.x == 0) p.tile[blockIdx.x] = n;
}

__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(const PagesDev p, int32_t *pairs, uint32_t max_pairs) {
    __shared__ uint32_t sums[32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    uint32_t low = 0, all = 0, n, u, ignored;
    int4 v = make_int4(0, 0, 0, 0);
    if (p.n_tiles <= SMALL) {
#pragma unroll
        for (uint32_t i = 0; i < SMALL; ++i) {
            const int4 x = i < p.n_tiles ? tile_counts(p, i, 0) : make_int4(0, 0, 0, 0);
            all += 4 - zeros(x);
            if (i < blockIdx.x) low += 4 - zeros(x);
            if (i == blockIdx.x) v = x;
        }
    } else {
        for (uint32_t i = threadIdx.x; i < p.n_tiles; i += PLAN_THREADS) {
            const uint32_t c = p.tile[i];
            all += c;
            if (i < blockIdx.x) low += c;
        }
        v = tile_counts(p, blockIdx.x, 0);
    }
    scan(all, sums, n);
    scan(low, sums, u);
    u += scan(4 - zeros(v), sums, ignored);
    if (n == p.n_blocks && blockIdx.x == 0 && threadIdx.x == 0) *p.moves = 0;
    const int count[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
        const uint32_t id = blockIdx.x * TILE + threadIdx.x * 4 + k;
        if (id >= p.n_blocks) break;
        if (id == n) *p.moves = n - u;
        const bool used = count[k] != 0;
        if (used && id >= n) {
            const uint32_t r = n - 1 - u;
            p.rank[id] = r;
            if (r < max_pairs) pairs[2 * (uint64_t)r] = (int32_t)id;
        } else if (!used && id < n) {
            const uint32_t r = id - u;
            if (r < max_pairs) pairs[2 * (uint64_t)r + 1] = (int32_t)id;
        }
        u += used;
    }
}

__global__ void __launch_bounds__(ROW_THREADS) compact_apply_kernel(const PagesDev p, const TablesDev t, int32_t *pairs, uint32_t max_pairs, uint32_t *n_pairs, uint32_t per) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t n = min(*p.moves, max_pairs);
    if (blockIdx.x >= per * t.n_seq) {          // the counts, and the pairs behind the last
        const uint32_t first = blockIdx.x - per * t.n_seq, ctas = gridDim.x - per * t.n_seq;
        if (first == 0 && threadIdx.x == 0) *n_pairs = n;
        for (uint64_t r = first * ROW_THREADS + threadIdx.x; r < max_pairs; r += (uint64_t)ctas * ROW_THREADS) {
            int2 *pair = reinterpret_cast<int2 *>(pairs) + r;
            if (r >= n) {
                *pair = make_int2(-1, -1);
                continue;
            }
            const int2 m = *pair;
            p.refs[m.y] = p.refs[m.x];
            p.refs[m.x] = 0;
        }
        return;
    }
    const uint32_t s = blockIdx.x / per, part = blockIdx.x % per;
    Row r;
    if (!row_view(t, s, r)) {
        if (part == 0 && threadIdx.x == 0) report(t.status, TUTTI_EINVAL);
        return;
    }
    for (uint32_t i = part * ROW_THREADS + threadIdx.x; i < r.held; i += per * ROW_THREADS) {
        const int32_t id = t.block_ids[r.b0 + i];
        if (id == -1) continue;
        if ((uint32_t)id >= p.n_blocks) {
            report(t.status, TUTTI_EFAULT);
            continue;
        }
        const uint32_t k = p.rank[id];          // of a block that does not move: of an earlier call, or none
        if (k < n && pairs[2 * (uint64_t)k] == id) t.block_ids[r.b0 + i] = pairs[2 * (uint64_t)k + 1];
    }
}

// CTAs a row, so that rows of average room are done in about one round and the GPU is filled a few times at most.
uint32_t ctas_a_row(uint32_t n_seq, uint32_t n_blk, uint32_t ids, int sms) {
    const uint32_t most = (uint32_t)sms * 8 / n_seq + 1, want = n_blk / n_seq / ids + 1;
    return most < want ? most : want;
}

}  // namespace

}  // namespace tutti

using namespace tutti;

struct tutti_pages {
    tutti_ctx *ctx;
    int device;
    PagesDev dev;
    // rows' arrays, two each (and tiles); writers; top; rank.  In pieces, because those below a megabyte are made in 15 us each instead of 400 and more.
    uint32_t *memory[6];
};

namespace {

int check_tables(const tutti_tables_t *t) {
    if (!t || t->n_seq > TUTTI_PAGES_MAX_SEQ || t->n_blk > 0x7fffffffu) return TUTTI_EINVAL;
    if (t->n_seq && (!t->blk_start || !t->len)) return TUTTI_EINVAL;
    if (t->n_blk && !t->block_ids) return TUTTI_EINVAL;
    if (((uint64_t)t->blk_start | (uint64_t)t->block_ids | (uint64_t)t->len | (uint64_t)t->status) & 3) return TUTTI_EINVAL;
    return TUTTI_OK;
}

// `n` 32-bit words in memory
struct Words {
    const void *at;
    uint64_t n;
};
bool lie_over(const Words &a, const Words &b) {
    const uint64_t x = (uint64_t)a.at, y = (uint64_t)b.at;
    return x && y && a.n && b.n && x < y + 4 * b.n && y < x + 4 * a.n;
}

TablesDev on_device(const tutti_pages *pages, const tutti_tables_t *t) {
    return TablesDev{t->n_seq, t->n_blk, tutti_ctx_geom_(pages->ctx)->block_tokens, t->blk_start, t->block_ids, t->len, t->status};
}

}  // namespace

extern "C" {

// What the calls refuse, from the arguments alone.
int tutti_fork_check_(const tutti_tables_t *from, const int32_t *parent, const tutti_tables_t *to, uint32_t move) {
    if (check_tables(from) || check_tables(to) || move > TUTTI_FORK_MOVE) return TUTTI_EINVAL;
    if (to->n_seq && (!parent || ((uint64_t)parent & 3))) return TUTTI_EINVAL;
    if ((from->block_ids && from->block_ids == to->block_ids) || (from->len && from->len == to->len)) return TUTTI_EINVAL;
    // what is written lies over nothing that is read, nor over each other (what is read may: both tables may have one blk_start)
    const Words ids{to->block_ids, to->n_blk}, len{to->len, to->n_seq};
    const Words read[] = {{from->block_ids, from->n_blk}, {from->len, from->n_seq}, {from->blk_start, (uint64_t)from->n_seq + 1},
                          {to->blk_start, (uint64_t)to->n_seq + 1}, {parent, to->n_seq}};
    for (const Words &r : read)
        if (lie_over(ids, r) || lie_over(len, r)) return TUTTI_EINVAL;
    return lie_over(ids, len) ? TUTTI_EINVAL : TUTTI_OK;
}
int tutti_extend_check_(const tutti_tables_t *t, const uint32_t *n_new, const int32_t *pairs) {
    if (check_tables(t) || (t->n_seq && (!n_new || !pairs)) || (((uint64_t)n_new | (uint64_t)pairs) & 3)) return TUTTI_EINVAL;
    return TUTTI_OK;
}
int tutti_compact_check_(const tutti_tables_t *t, const int32_t *pairs, uint32_t max_pairs, const uint32_t *n_pairs) {
    if (check_tables(t) || !n_pairs || ((uint64_t)n_pairs & 3) || max_pairs > 0x7fffffffu) return TUTTI_EINVAL;
    if (max_pairs && (!pairs || ((uint64_t)pairs & 7))) return TUTTI_EINVAL;
    return TUTTI_OK;
}
int tutti_tables_check_(const tutti_tables_t *t) { return check_tables(t); }
int tutti_fork_given_back_(int now, int sum) { return given_back(now, sum); }

int tutti_pages_create(tutti_ctx_t *ctx, int32_t *refs, uint64_t n_blocks, tutti_pages_t **out) {
    if (!ctx || !refs || ((uint64_t)refs & 15) || !n_blocks || n_blocks > 0x7fffffffull || !out) return TUTTI_EINVAL;
    OnDevice on(tutti_ctx_device_(ctx));
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    tutti_pages *p = new (std::nothrow) tutti_pages();
    if (!p) return TUTTI_ENOMEM;
    const uint32_t tiles = (uint32_t)((n_blocks + TILE - 1) / TILE);
    const size_t rows = 2 * (size_t)TUTTI_PAGES_MAX_SEQ, words[6] = {rows + 32 + tiles, rows, rows, n_blocks, n_blocks, (size_t)tiles * TILE};
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < 6; ++i) {
        p->memory[i] = nullptr;
        if (e == cudaSuccess) e = cudaMalloc((void **)&p->memory[i], words[i] * 4);
        if (e == cudaSuccess) e = cudaMemset(p->memory[i], 0, words[i] * 4);
    }
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        for (uint32_t *m : p->memory)
            if (m) cudaFree(m);
        delete p;
        fail(e, "workspace of the pages");
        return TUTTI_ENOMEM;
    }
    p->ctx = ctx;
    p->device = tutti_ctx_device_(ctx);
    PagesDev &d = p->dev;
    d.refs = refs;
    d.n_blocks = (uint32_t)n_blocks;
    d.n_tiles = tiles;
    d.turn = p->memory[0];
    d.begin = d.turn + TUTTI_PAGES_MAX_SEQ;
    d.arrive = p->memory[0] + rows;
    d.moves = d.arrive + 1;
    d.total = (unsigned long long *)(d.arrive + 2);
    d.tile = d.arrive + 32;
    d.entry = p->memory[1];
    d.mark = (int32_t *)d.entry + TUTTI_PAGES_MAX_SEQ;
    d.keep_id = (int32_t *)p->memory[2];
    d.keep_count = d.keep_id + TUTTI_PAGES_MAX_SEQ;
    d.writers = p->memory[3];
    d.top = p->memory[4];
    d.rank = p->memory[5];
    *out = p;
    return TUTTI_OK;
}

int tutti_pages_destroy(tutti_pages_t *p) {
    if (!p) return TUTTI_EINVAL;
    OnDevice on(p->device);
    cudaDeviceSynchronize();
    for (uint32_t *m : p->memory) cudaFree(m);
    delete p;
    return TUTTI_OK;
}

int tutti_pages_fork(tutti_pages_t *pages, const tutti_tables_t *from, const int32_t *parent, const tutti_tables_t *to, uint32_t move, void *stream) {
    if (!pages) return TUTTI_EINVAL;
    if (int rc = tutti_fork_check_(from, parent, to, move)) return rc;
    const uint32_t rows = from->n_seq + to->n_seq;
    if (!rows) return TUTTI_OK;
    OnDevice on(pages->device);
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    const uint32_t groups = (from->n_seq + GROUP - 1) / GROUP;
    const uint32_t per = ctas_a_row(rows, from->n_blk / 2 + to->n_blk / 2, ROW_IDS, tutti_ctx_sms_(pages->ctx));
    const uint32_t segs = groups ? ctas_a_row(groups, from->n_blk / GROUP, ROW_THREADS, tutti_ctx_sms_(pages->ctx)) : 0;
    const cudaError_t e = launch_behind(fork_kernel, per * to->n_seq + segs * groups, ROW_THREADS, 0, (cudaStream_t)stream, pages->dev, on_device(pages, from), parent, on_device(pages, to), move, per, segs);
    return e == cudaSuccess ? TUTTI_OK : fail(e, "fork launch");
}

int tutti_pages_extend(tutti_pages_t *pages, const tutti_tables_t *t, const uint32_t *n_new, int32_t *pairs, void *stream) {
    if (!pages) return TUTTI_EINVAL;
    if (int rc = tutti_extend_check_(t, n_new, pairs)) return rc;
    if (!t->n_seq) return TUTTI_OK;
    OnDevice on(pages->device);
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    const cudaError_t e = launch_behind(extend_kernel, pages->dev.n_tiles + 1, PLAN_THREADS, 0, (cudaStream_t)stream, pages->dev, on_device(pages, t), n_new, pairs);
    return e == cudaSuccess ? TUTTI_OK : fail(e, "extend launch");
}

int tutti_pages_release(tutti_pages_t *pages, const tutti_tables_t *t, const uint8_t *which, void *stream) {
    if (!pages) return TUTTI_EINVAL;
    if (int rc = check_tables(t)) return rc;
    if (!t->n_seq) return TUTTI_OK;
    OnDevice on(pages->device);
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    const uint32_t per = ctas_a_row(t->n_seq, t->n_blk, ROW_THREADS, tutti_ctx_sms_(pages->ctx));
    const cudaError_t e = launch_behind(release_kernel, per * t->n_seq, ROW_THREADS, 0, (cudaStream_t)stream, pages->dev, on_device(pages, t), which, per);
    return e == cudaSuccess ? TUTTI_OK : fail(e, "release launch");
}

int tutti_pages_trim(tutti_pages_t *pages, const tutti_tables_t *t, const tutti_window_t *window, void *stream) {
    if (!pages) return TUTTI_EINVAL;
    if (int rc = check_tables(t)) return rc;
    if (int rc = tutti_window_check_(window)) return rc;
    if (!t->n_seq) return TUTTI_OK;
    OnDevice on(pages->device);
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    const uint32_t per = ctas_a_row(t->n_seq, t->n_blk, ROW_THREADS, tutti_ctx_sms_(pages->ctx));
    const cudaError_t e = launch_behind(trim_kernel, per * t->n_seq, ROW_THREADS, 0, (cudaStream_t)stream, pages->dev, on_device(pages, t), window->window, window->sinks, per);
    return e == cudaSuccess ? TUTTI_OK : fail(e, "trim launch");
}

int tutti_pages_compact(tutti_pages_t *pages, const tutti_tables_t *t, int32_t *pairs, uint32_t max_pairs, uint32_t *n_pairs, void *stream) {
    if (!pages) return TUTTI_EINVAL;
    if (int rc = tutti_compact_check_(t, pairs, max_pairs, n_pairs)) return rc;
    OnDevice on(pages->device);
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    const PagesDev &d = pages->dev;
    const int sms = tutti_ctx_sms_(pages->ctx);
    const uint32_t per = t->n_seq ? ctas_a_row(t->n_seq, t->n_blk, ROW_THREADS, sms) : 1;
    const uint32_t movers = max_pairs / ROW_THREADS + 1 < (uint32_t)sms ? max_pairs / ROW_THREADS + 1 : (uint32_t)sms;
    cudaError_t e = cudaSuccess;
    if (d.n_tiles > SMALL) e = launch_behind(compact_count_kernel, d.n_tiles, PLAN_THREADS, 0, (cudaStream_t)stream, d);
    if (e == cudaSuccess) e = launch_behind(compact_plan_kernel, d.n_tiles, PLAN_THREADS, 0, (cudaStream_t)stream, d, pairs, max_pairs);
    if (e == cudaSuccess) e = launch_behind(compact_apply_kernel, per * t->n_seq + movers, ROW_THREADS, 0, (cudaStream_t)stream, d, on_device(pages, t), pairs, max_pairs, n_pairs, per);
    return e == cudaSuccess ? TUTTI_OK : fail(e, "compact launch");
}

}  // extern "C"
