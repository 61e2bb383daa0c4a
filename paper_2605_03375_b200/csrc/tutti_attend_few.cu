// Attention of few rows per sequence (a decode step).  Bound: HBM, the cache is read once.
// On a B200 (6.45 TB/s copy), the kernel alone, 128-wide heads: 64 ragged requests on 1-token pages (2.3 GB) 360 us =
// 6.4 TB/s; one of 131072 tokens (0.54 GB) 92 us = 5.8 TB/s; 8 of 32768, 8-bit (0.54 GB), 110 us = 4.9
// TB/s; 64-wide heads, 16-bit, 48 ragged (0.44 GB), 87 us = 5.0 TB/s; 64-wide heads, 8-bit, 48 ragged (0.22 GB), 70 us = 3.1 TB/s (bound by instructions: 17 a byte).  One
// request of 1 / 512 / 4096 tokens 5.2 / 9.0 / 12.5 us: three rounds of dependent loads, and the join.
// Under a window (WIN) the units between a sequence's first tokens and its window are left out: 64 ragged requests that see 4096
// keys (1.04 GB) 163 us = 6.4 TB/s, on 1-token pages 171 us, 8-bit 113 us = 4.6 TB/s.
#include <type_traits>

#include "tutti_attend.h"

namespace tutti {

namespace {

// ---------------------------------------------------------------------------------------------
// Few rows per sequence (decode): one pass over the cache at HBM speed.
//
// A *tile* is 8 or 16 rows of one sequence and KV head: (new token, query head of the group) pairs,
// one or two B fragments of the warp-level matrix instruction.  Its keys are cut into units of WARPS x KW
// keys; all units of all tiles of the step, laid end to end, are dealt out evenly over a fixed
// number of workers (CTAs), so ragged batches, one long sequence and captured graphs whose lengths
// change all load every SM alike and the host needs no length.  A worker's share is a run of
// units: at most its first and its last tile are shared with neighbours.  Those parts go to the
// workspace (two slots a worker) and whoever arrives last at a tile joins its parts in worker
// order: the result does not depend on the order of arrival.
//
// Inside a worker each warp takes KW keys of a unit on its own: gather through the block table
// with cp.async into its ring of STAGES stages (a row of one head is the largest piece that is
// contiguous in every pool layout), S^T = K Q^T, running maximum and sum, O^T += V^T P^T, all in
// registers; no CTA barrier until a tile ends.  Keys and values are the A operand, so that the
// few rows fill the N of 8 of one instruction: half the instructions and registers of the other
// way round.  8-bit caches are multiplied as f16 codes (exact); the scale of a key goes onto
// its score, the scale of a value onto its probability.
constexpr int WARPS = 4;
// _8: 8-bit caches (the ring and the workers: with 8 rows), see below.
constexpr int STAGES = 3, STAGES_8 = 2;     // of a warp's ring
constexpr uint32_t BYTES_8 = 8192;          // of a stage
constexpr int WORKERS_8 = 3;                // an SM
constexpr int DEEP = 16, DEEP_8 = 4;        // parts whose loads are in flight while a tile is joined (registers: 16 cost
                                            // the 8-bit loop 4 %)
constexpr int MIN_UNITS = 2;                // of a worker that takes a part of a tile: joining the parts costs, too

__device__ inline void ldm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ inline void ldm4t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ inline void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ inline void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// an 8 x 8 block of 16-bit elements, thread (g, c) holding row g, columns 2 c and 2 c + 1
__device__ inline uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// A place in the step's units laid end to end: unit u of row tile r and KV head h of sequence s.
struct Place {
    uint32_t s, h, r, u;
    uint32_t n_tiles, n_units;      // of the sequence: row tiles, units of each
    SeqView v;
};
// WIN: units that no row of the sequence sees, between its first tokens and its window, are left out.
template <bool WIN>
struct Cursor : Place {};
template <>
struct Cursor<true> : Place {
    uint32_t gap;                   // how many
};
__device__ inline uint32_t sink_units(const AttendParams &p, uint32_t unit_keys) { return (p.sinks + unit_keys - 1) / unit_keys; }

// Row tiles and units of a sequence (0 tiles: nothing to do); the error code, if any.
template <bool WIN>
__device__ inline int seq_shape(const AttendParams &p, uint32_t rows, uint32_t unit_keys, uint32_t s, Cursor<WIN> &k) {
    const int code = seq_view(p.step, p.pool.block_tokens, s, k.v);
    k.n_tiles = code == TUTTI_OK ? (k.v.n_new * p.group + rows - 1) / rows : 0;
    k.n_units = code == TUTTI_OK && k.v.ctx ? (k.v.ctx + unit_keys - 1) / unit_keys : 1;
    if constexpr (WIN) {
        const int64_t start = p.window_start((int64_t)k.v.ctx - k.v.n_new);
        const uint32_t behind = start > 0 ? (uint32_t)start / unit_keys : 0, front = sink_units(p, unit_keys);
        k.gap = code == TUTTI_OK && behind > front ? behind - front : 0;
        k.n_units -= k.gap;
    }
    return code;
}
// Which unit of the sequence's keys unit u is.
template <bool WIN>
__device__ inline uint32_t key_unit(const AttendParams &p, uint32_t unit_keys, const Cursor<WIN> &k) {
    if constexpr (WIN) return k.u + (k.u >= sink_units(p, unit_keys) ? k.gap : 0);
    else return k.u;
}

template <bool WIN>
__device__ inline void advance(const AttendParams &p, uint32_t rows, uint32_t unit_keys, Cursor<WIN> &k) {
    if (++k.u < k.n_units) return;
    k.u = 0;
    if (++k.r < k.n_tiles) return;
    k.r = 0;
    if (++k.h < p.pool.n_kv_heads) return;
    k.h = 0;
    do {
        if (++k.s >= p.step.n_seq) return;      // behind the last unit: not used
        seq_shape(p, rows, unit_keys, k.s, k);
    } while (k.n_tiles == 0);
}

// Q, K and V have the type T; 8-bit caches (C8) are multiplied as f16.  NB: blocks of 8 rows.
template <typename T, bool C8, int D, int NB>
struct Few {
    using M = typename std::conditional<C8, __half, T>::type;        // type of the matrix instructions
    static constexpr int ROWS = 8 * NB;
    // 8-bit caches take more instructions a byte (widening): with 8 rows 168 registers are enough for
    // 12 warps an SM instead of 8, each with a stage less (8 x 32768 keys: 108 us with 2 or 3 workers of
    // 32 keys a step, 131-135 us with 3 or 4 of 16; 64-wide heads, ragged: 73 with 3, 81 with 2).
    static constexpr int WORKERS_PER_SM = C8 && NB == 1 ? WORKERS_8 : 2;
    static constexpr int STAGES = C8 && NB == 1 ? STAGES_8 : tutti::STAGES;
    static constexpr uint32_t STAGE_BYTES = C8 && NB == 1 ? BYTES_8 : 8192;  // keys and values of one warp's KW keys
    static constexpr int RB = D * (C8 ? 1 : 2);                      // bytes of a row
    static constexpr int KW = STAGE_BYTES / (2 * RB);                // keys of a warp's step
    static constexpr int UNIT = WARPS * KW;
    static constexpr int MT = KW / 16;                               // blocks of 16 keys
    static constexpr int DT = D / 16;                                // blocks of 16 dimensions
    static constexpr int KPL = (KW + 31) / 32;                       // keys whose address a lane knows
    static constexpr int CH = RB / 16;                               // 16-byte chunks of a row
    static constexpr uint32_t SCALES = C8 ? KW * 8 : 0;              // scales of the stage's keys, then values
    static constexpr uint32_t STAGE = STAGE_BYTES + SCALES;
    // f16 probabilities are kept 2^OFF times too large: full precision down to 2^-28 of the largest
    // instead of 2^-14.  (8-bit: the products with the value scales are, see `unit` below.)
    static constexpr float OFF = std::is_same<M, __half>::value && !C8 ? 14.0f : 0.0f;
    static constexpr float UP = 16384.0f;
    static constexpr uint32_t OFF_MASK = WARPS * STAGES * STAGE;     // uint64 keys that exist, by warp and stage
    static constexpr uint32_t OFF_ML = OFF_MASK + WARPS * STAGES * 8;
    static constexpr uint32_t OFF_PLAN = OFF_ML + WARPS * ROWS * 8;
    static constexpr uint32_t SMEM = OFF_PLAN + 128;
    static_assert(STAGE_BYTES >= ROWS * D * 4, "a warp's sums go through one of its stages");

    // Where 16-byte chunk `ch` of row `row` lies: rotated so that the loads below meet no bank twice.
    __device__ static uint32_t place(uint32_t row, uint32_t ch, bool value) {
        if (!C8) return row * RB + ((ch ^ (row & 7)) * 16);
        if (RB == 64) return (row / 2) * 128 + ((((row & 1) * 4 + ch) ^ ((row >> 1 & 3) << 1)) * 16);
        return row * RB + ((ch ^ (value ? (row >> 1 & 3) << 1 : (row & 1) << 2)) * 16);
    }
};

template <typename T, bool C8, int D, int NB, bool WIN>
__global__ void __launch_bounds__(WARPS * 32, Few<T, C8, D, NB>::WORKERS_PER_SM)
attend_few_kernel(const __grid_constant__ AttendParams p, const Workspace ws) {
    using F = Few<T, C8, D, NB>;
    using M = typename F::M;
    if constexpr (WIN) asm volatile("griddepcontrol.wait;" ::: "memory");
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane / 4, c = lane % 4;
    unsigned char *ring = smem + warp * F::STAGES * F::STAGE;
    uint64_t *exists = reinterpret_cast<uint64_t *>(smem + F::OFF_MASK) + warp * F::STAGES;
    float2 *ml = reinterpret_cast<float2 *>(smem + F::OFF_ML);
    uint32_t *plan = reinterpret_cast<uint32_t *>(smem + F::OFF_PLAN);

    // ---- this worker's share: a prefix sum over the sequences' units ----
    const uint32_t per = (p.step.n_seq + WARPS * 32 - 1) / (WARPS * 32);
    unsigned long long mine = 0;
    uint32_t my_tiles = 0;
    Cursor<WIN> own;                               // the thread's last sequence (its only one, mostly)
    own.s = ~0u;
    for (uint32_t s = threadIdx.x * per; s < min((threadIdx.x + 1) * per, p.step.n_seq); ++s) {
        const int code = seq_shape(p, F::ROWS, F::UNIT, s, own);
        own.s = s;
        if (code != TUTTI_OK && blockIdx.x == 0) report(p.step, code);
        mine += (unsigned long long)own.n_tiles * own.n_units * p.pool.n_kv_heads;
        my_tiles += own.n_tiles * p.pool.n_kv_heads;
    }
    unsigned long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    unsigned long long *sums = reinterpret_cast<unsigned long long *>(plan);
    my_tiles = __reduce_add_sync(0xffffffffu, my_tiles);
    if (lane == 31) sums[warp] = incl, plan[2 * WARPS + warp] = my_tiles;
    __syncthreads();
    uint32_t tiles = 0;
    unsigned long long total = 0, before = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        if (i < (int)warp) before += sums[i];
        total += sums[i];
        tiles += plan[2 * WARPS + i];
    }
    unsigned long long workers = (total + MIN_UNITS - 1) / MIN_UNITS;
    if (workers < tiles) workers = tiles;
    if (workers > ws.workers) workers = ws.workers;
    const uint32_t w = blockIdx.x;
    if (w >= workers) return;
    const unsigned long long x0 = quotient(w * total, workers), x1 = quotient((w + 1) * total, workers);
    before += incl - mine;
    __syncthreads();
    if (x0 >= before && x0 < before + mine) {      // one thread's sequences hold the first unit
        unsigned long long at = before;
        for (uint32_t s = threadIdx.x * per;; ++s) {
            if (s != own.s) seq_shape(p, F::ROWS, F::UNIT, s, own);
            const unsigned long long n = (unsigned long long)own.n_tiles * own.n_units * p.pool.n_kv_heads;
            if (x0 < at + n) {
                own.s = s;
                const unsigned long long tile = quotient(x0 - at, own.n_units);
                own.h = (uint32_t)quotient(tile, own.n_tiles);
                own.r = (uint32_t)(tile - (unsigned long long)own.h * own.n_tiles);
                own.u = (uint32_t)(x0 - at - tile * own.n_units);
                *reinterpret_cast<Cursor<WIN> *>(plan) = own;
                break;
            }
            at += n;
            own.s = ~0u;
        }
    }
    __syncthreads();
    Cursor<WIN> get = *reinterpret_cast<const Cursor<WIN> *>(plan);

    // ---- gathering ----
    // The ids of a unit's blocks are looked up two units before its rows are fetched, and not touched
    // until then (the first use waits for the load).
    struct Pending {
        uint32_t key0, ctx, h;                     // of a unit: the warp's first key, keys that exist, KV head
        uint32_t start;                            // WIN: keys from here on, and the first p.sinks, are seen
        int32_t id[F::KPL];                        // of the lane's keys
    } pend[2];
    auto in_sight = [&](const Pending &u, uint32_t key) { return key < u.ctx && (!WIN || key < p.sinks || key >= u.start); };
    Cursor<WIN> look = get;
    unsigned long long look_x = x0, put_x = x0;
    auto locate = [&](Pending &u) {
        u.key0 = (key_unit(p, F::UNIT, look) * WARPS + warp) * F::KW;
        u.ctx = look.v.ctx;
        if constexpr (WIN) {
            const int64_t start = p.window_start((int64_t)look.v.ctx - look.v.n_new);
            u.start = start > 0 ? (uint32_t)start : 0;
        }
        u.h = look.h;
        if (look_x < x1) {
#pragma unroll
            for (int i = 0; i < F::KPL; ++i) {
                const uint32_t key = u.key0 + i * 32 + lane;
                u.id[i] = -1;
                if (i * 32 + lane < F::KW && in_sight(u, key)) u.id[i] = __ldg(p.step.block_ids + look.v.b0 + p.pool.block_of(key));
            }
            advance(p, F::ROWS, F::UNIT, look);
        }
        ++look_x;
    };
    locate(pend[0]);
    locate(pend[1]);
    auto fetch = [&](uint32_t stage) {             // issues the loads of the next unit, then looks up the ids two behind
        if (put_x < x1) {
            unsigned char *st = ring + stage * F::STAGE;
            const uint32_t kst = smem_addr(st), vst = kst + F::KW * F::RB;
            const Pending &u = pend[0];
            uint64_t mask = 0;
            int64_t off[F::KPL];
#pragma unroll
            for (int i = 0; i < F::KPL; ++i) {
                const uint32_t key = u.key0 + i * 32 + lane;
                const bool held = i * 32 + lane < F::KW && in_sight(u, key), ok = held && (uint32_t)u.id[i] < p.pool.n_blocks;
                if (held && !ok) report(p.step, TUTTI_EFAULT);
                mask |= (uint64_t)__ballot_sync(0xffffffffu, ok) << (32 * i);
                if (C8 && i * 32 + lane < F::KW) {
                    const uint64_t at = ok ? (uint64_t)(uint32_t)u.id[i] * p.pool.scale_row + u.h : 0;
                    cp4(kst + F::STAGE_BYTES + (i * 32 + lane) * 4, p.pool.k_scale + at, ok);
                    cp4(kst + F::STAGE_BYTES + (F::KW + i * 32 + lane) * 4, p.pool.v_scale + at, ok);
                }
                off[i] = ok ? block_offset(p.pool, u.id[i]) + (int64_t)(p.pool.row_of(key) * p.pool.tok_stride + u.h * p.pool.head_stride) : -1;
            }
            if (lane == 0) exists[stage] = mask;
#pragma unroll
            for (int i = 0; i < F::KW * F::CH / 32; ++i) {
                const uint32_t row = (i * 32 + lane) / F::CH, ch = lane % F::CH;
                const int64_t o = __shfl_sync(0xffffffffu, off[(i * 32 / F::CH) / 32], row % 32);
                const bool ok = o >= 0;
                const uint64_t a = (ok ? (uint64_t)o : 0) + ch * 16;
                cp16(kst + F::place(row, ch, false), (const void *)(p.pool.k_base + a), ok);
                cp16(vst + F::place(row, ch, true), (const void *)(p.pool.v_base + a), ok);
            }
            ++put_x;
            pend[0] = pend[1];
            locate(pend[1]);
        }
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < F::STAGES - 1; ++i) fetch(i);

    // ---- the worker's tiles ----
    // The division by the group, a few times a tile, as a product on 8-bit caches only: on 16-bit ones the
    // code that the compiler then makes of the loop is 10 % slower (1-token pages 399 us against 361; 8-bit
    // the other way round, 70 against 75).
    auto token_of = [&](uint32_t row) { return C8 ? p.token_of(row) : row / p.group; };
    uint32_t stage = 0;
    for (unsigned long long x = x0; x < x1;) {
        const uint32_t h = get.h, row0 = get.r * F::ROWS;
        const uint32_t n_rows = get.v.n_new * p.group;
        const int64_t first = (int64_t)get.v.ctx - get.v.n_new;
        const unsigned long long tile0 = x - get.u;                       // the tile's units: [tile0, tile0 + n_units)
        const unsigned long long seg_end = min(x1, tile0 + get.n_units);
        // Query fragments: row g of each block of 8.  Scores: rows 2 c and 2 c + 1 of each block, their
        // positions (the last key they see) and factors.
        int64_t pos[NB][2];
        float rowscale[NB][2];
        uint32_t qf[NB][D / 16][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t row = row0 + b * 8 + g;
            const bool ok = row < n_rows;
            const uint32_t i = ok ? token_of(row) : 0, qh = h * p.group + (ok ? row - i * p.group : 0);
            const T *q = (const T *)p.q + (uint64_t)(get.v.q0 + i) * p.q_stride + (uint64_t)qh * D;
            float mul = p.scale * 1.4426950408889634f;
            if constexpr (!C8) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        qf[b][k][j] = ok ? *reinterpret_cast<const uint32_t *>(q + k * 16 + j * 8 + 2 * c) : 0;
            } else {
                // the k index of a step is permuted: a thread's 16 elements are 16 neighbouring dimensions
                float e16[D / 4], top = 0;
#pragma unroll
                for (int d = 0; d < D / 64; ++d) {
                    uint4 u[2] = {};
                    if (ok) {
                        u[0] = *reinterpret_cast<const uint4 *>(q + d * 64 + c * 16);
                        u[1] = *reinterpret_cast<const uint4 *>(q + d * 64 + c * 16 + 8);
                    }
                    const T *e = reinterpret_cast<const T *>(u);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        e16[d * 16 + j] = (float)e[j];
                        top = fmaxf(top, fabsf(e16[d * 16 + j]));
                    }
                }
                // a row of bf16 queries is scaled by a power of two so that f16, the type that holds the codes, holds
                // it: exactly, but for elements below 2^-14 of the row's largest, which keep an error of 2^-25 of it
                float down = 1.0f;
                if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -60), 126);
                    down = __uint_as_float((uint32_t)(127 - e) << 23);
                    mul *= __uint_as_float((uint32_t)(127 + e) << 23);
                }
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int at = (k / 4) * 16 + (k % 4) * 4 + 2 * j;
                        qf[b][k][j] = pack2(e16[at] * down, e16[at + 1] * down, __half());
                    }
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const uint32_t mine = row0 + b * 8 + 2 * c + r;
                pos[b][r] = mine < n_rows ? first + token_of(mine) : -1;
                rowscale[b][r] = __shfl_sync(0xffffffffu, mul, (2 * c + r) * 4);
            }
        }
        float o[NB][F::DT][4], m[NB][2], l[NB][2];
        // 8-bit: a row's O is kept in units of a power of two near its largest product of probability and
        // value scale so far, so that the f16 products hold what counts in the row whatever the
        // scales of other blocks are.
        float unit[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            unit[b][0] = unit[b][1] = 0;
            m[b][0] = m[b][1] = -INFINITY;
            l[b][0] = l[b][1] = 0;
#pragma unroll
            for (int i = 0; i < F::DT; ++i) o[b][i][0] = o[b][i][1] = o[b][i][2] = o[b][i][3] = 0;
        }
        const int64_t last_all = first + token_of(row0);        // keys up to here are seen by every row of the tile
        const int64_t hidden = WIN ? first + token_of(min(row0 + F::ROWS, n_rows) - 1) - p.window : 0;      // up to here not by every one

        for (; x < seg_end; ++x) {
            cp_wait<F::STAGES - 2>();
            __syncwarp();
            fetch(stage == 0 ? F::STAGES - 1 : stage - 1);      // the stage before this one is free
            unsigned char *st = ring + stage * F::STAGE;
            const uint32_t kst = smem_addr(st), vst = kst + F::KW * F::RB;
            const uint64_t there = exists[stage];
            const int64_t key0 = (int64_t)(key_unit(p, F::UNIT, get) * WARPS + warp) * F::KW;
            constexpr uint64_t ALL = F::KW == 64 ? ~0ull : (1ull << (F::KW & 63)) - 1;
            if (there) {
                // scores: fragment element e is key 16 t + g + 8 (e / 2), row 2 c + e % 2
                float s[NB][F::MT][4];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int t = 0; t < F::MT; ++t) s[b][t][0] = s[b][t][1] = s[b][t][2] = s[b][t][3] = 0;
#pragma unroll
                for (int t = 0; t < F::MT; ++t) {
                    if constexpr (!C8) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            uint32_t a[4];
                            ldm4(a, kst + F::place(t * 16 + (lane & 15), k * 2 + (lane >> 4), false));
#pragma unroll
                            for (int b = 0; b < NB; ++b) mma(s[b][t], a, qf[b][k][0], qf[b][k][1], M());
                        }
                    } else {
#pragma unroll
                        for (int d = 0; d < D / 64; ++d) {
                            const uint4 u = *reinterpret_cast<const uint4 *>(st + F::place(t * 16 + g, d * 4 + c, false));
                            const uint4 v = *reinterpret_cast<const uint4 *>(st + F::place(t * 16 + g + 8, d * 4 + c, false));
                            const uint32_t lo[4] = {u.x, u.y, u.z, u.w}, hi[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                uint32_t a[4];
                                codes4(lo[k], a[0], a[2]);
                                codes4(hi[k], a[1], a[3]);
#pragma unroll
                                for (int b = 0; b < NB; ++b) mma(s[b][t], a, qf[b][d * 4 + k][0], qf[b][d * 4 + k][1], M());
                            }
                        }
                    }
                }
                const bool masked = there != ALL || key0 + F::KW - 1 > last_all || (WIN && key0 <= hidden);
                float vs[F::MT][2];                      // 8-bit: value scales of the lane's keys
                if constexpr (C8) {
#pragma unroll
                    for (int t = 0; t < F::MT; ++t)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            vs[t][i] = *reinterpret_cast<const float *>(st + F::STAGE_BYTES + (F::KW + t * 16 + g + 8 * i) * 4);
                }
                uint32_t pf[NB][F::MT][2];
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int t = 0; t < F::MT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float ks = rowscale[b][e & 1];
                            const int key = t * 16 + g + 8 * (e / 2);
                            if constexpr (C8) ks *= *reinterpret_cast<const float *>(st + F::STAGE_BYTES + key * 4);
                            s[b][t][e] *= ks;
                            if (masked && (!(there >> key & 1) || key0 + key > pos[b][e & 1] ||
                                           (WIN && key0 + key <= pos[b][e & 1] - p.window && key0 + key >= p.sinks)))
                                s[b][t][e] = -INFINITY;
                            top[e & 1] = fmaxf(top[e & 1], s[b][t][e]);
                        }
                    float alpha[2], sub[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 4));
                        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 8));
                        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 16));
                        const float m2 = fmaxf(m[b][r], top[r]);
                        sub[r] = m2 == -INFINITY ? 0 : m2;       // a row that has seen nothing yet
                        alpha[r] = ex2(m[b][r] - sub[r]);
                        m[b][r] = m2;
                        l[b][r] *= alpha[r];
                        sub[r] -= F::OFF;
                    }
                    float up[2] = {1.0f, 1.0f}, most[2] = {0, 0};
#pragma unroll
                    for (int t = 0; t < F::MT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[b][t][e] = ex2(s[b][t][e] - sub[e & 1]);
                            l[b][e & 1] += s[b][t][e];
                            if constexpr (C8) {
                                s[b][t][e] *= vs[t][e / 2];
                                most[e & 1] = fmaxf(most[e & 1], fabsf(s[b][t][e]));
                            }
                        }
                    if constexpr (C8) {
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            most[r] = fmaxf(most[r], __shfl_xor_sync(0xffffffffu, most[r], 4));
                            most[r] = fmaxf(most[r], __shfl_xor_sync(0xffffffffu, most[r], 8));
                            most[r] = fmaxf(most[r], __shfl_xor_sync(0xffffffffu, most[r], 16));
                            most[r] = fmaxf(most[r], unit[b][r] * alpha[r]);
                            // the power of two at or below it, between 2^-100 and 2^126
                            const float next = __uint_as_float(min(max(__float_as_uint(most[r]) >> 23, 27u), 253u) << 23);
                            alpha[r] *= unit[b][r] / next;
                            unit[b][r] = next;
                            up[r] = F::UP / next;
                        }
                    }
                    if (__any_sync(0xffffffffu, alpha[0] != 1.0f || alpha[1] != 1.0f)) {
#pragma unroll
                        for (int i = 0; i < F::DT; ++i) {
                            o[b][i][0] *= alpha[0];
                            o[b][i][1] *= alpha[1];
                            o[b][i][2] *= alpha[0];
                            o[b][i][3] *= alpha[1];
                        }
                    }
                    // From (key g, rows 2 c and 2 c + 1) to (row g, keys 2 c and 2 c + 1).  Probabilities are rounded to 16
                    // bits, the type of the matrix instruction; l has summed them in 32.
#pragma unroll
                    for (int t = 0; t < F::MT; ++t)
#pragma unroll
                        for (int i = 0; i < 2; ++i) pf[b][t][i] = transpose8(pack2(s[b][t][2 * i] * up[0], s[b][t][2 * i + 1] * up[1], M()));
                }
                // values
#pragma unroll
                for (int t = 0; t < F::MT; ++t) {
                    if constexpr (!C8) {
#pragma unroll
                        for (int i = 0; i < F::DT; ++i) {
                            uint32_t a[4];
                            ldm4t(a, vst + F::place(t * 16 + (lane & 7) + (lane >> 4) * 8, i * 2 + (lane >> 3 & 1), true));
#pragma unroll
                            for (int b = 0; b < NB; ++b) mma(o[b][i], a, pf[b][t][0], pf[b][t][1], M());
                        }
                    } else {
                        // rows g and g + 8 of fragment i are dimensions g * D / 8 + 2 i and + 1: a thread's codes of a key
                        // are neighbours
                        const unsigned char *vrow = st + F::KW * F::RB;
                        uint32_t word[4][D / 32];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t row = t * 16 + 2 * c + (j & 1) + (j >> 1) * 8;
                            if constexpr (D == 128) {
                                const uint4 u = *reinterpret_cast<const uint4 *>(vrow + F::place(row, g, true));
                                word[j][0] = u.x, word[j][1] = u.y, word[j][2] = u.z, word[j][3] = u.w;
                            } else {
                                const uint2 u = *reinterpret_cast<const uint2 *>(vrow + F::place(row, g / 2, true) + (g & 1) * 8);
                                word[j][0] = u.x, word[j][1] = u.y;
                            }
                        }
#pragma unroll
                        for (int i = 0; i < F::DT; ++i) {
                            const uint32_t pick = i & 1 ? 0x7362 : 0x5140;       // two neighbouring dimensions of two keys
                            uint32_t a[4];
                            codes4(__byte_perm(word[0][i / 2], word[1][i / 2], pick), a[0], a[1]);
                            codes4(__byte_perm(word[2][i / 2], word[3][i / 2], pick), a[2], a[3]);
#pragma unroll
                            for (int b = 0; b < NB; ++b) mma(o[b][i], a, pf[b][t][0], pf[b][t][1], M());
                        }
                    }
                }
            }
            __syncwarp();
            if (x + 1 < seg_end) {
                stage = stage + 1 == F::STAGES ? 0 : stage + 1;
                ++get.u;
            }
        }

        // ---- join the warps: O goes through the stage just used, which no load is aimed at ----
        const bool whole = get.u + 1 == get.n_units && tile0 >= x0;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                l[b][r] += __shfl_xor_sync(0xffffffffu, l[b][r], 4);
                l[b][r] += __shfl_xor_sync(0xffffffffu, l[b][r], 8);
                l[b][r] += __shfl_xor_sync(0xffffffffu, l[b][r], 16);
                if (g == 0) ml[warp * F::ROWS + b * 8 + 2 * c + r] = make_float2(m[b][r], l[b][r]);
            }
        __syncthreads();
        float *mine_o = reinterpret_cast<float *>(ring + stage * F::STAGE);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const uint32_t row = b * 8 + 2 * c + r;
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < WARPS; ++i) top = fmaxf(top, ml[i * F::ROWS + row].x);
                const float f = top == -INFINITY ? 0 : ex2(m[b][r] - top) * (C8 ? unit[b][r] * (1.0f / F::UP) : 1.0f);
                float *dst = mine_o + row * D;
#pragma unroll
                for (int i = 0; i < F::DT; ++i) {
                    const uint32_t d0 = C8 ? g * (D / 8) + 2 * i : i * 16 + g, d1 = C8 ? d0 + 1 : d0 + 8;
                    dst[d0 ^ (c * 8)] = o[b][i][r] * f;
                    dst[d1 ^ (c * 8)] = o[b][i][2 + r] * f;
                }
            }
        __syncthreads();
        // TPR threads a row, each every TPR-th group of four dimensions
        constexpr int TPR = WARPS * 32 / F::ROWS, GROUPS = D / 4 / TPR;
        const uint32_t row = threadIdx.x / TPR, lanec = threadIdx.x % TPR;
        float M_ = -INFINITY, L = 0;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) M_ = fmaxf(M_, ml[i * F::ROWS + row].x);
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            const float2 e = ml[i * F::ROWS + row];
            L += e.y * (M_ == -INFINITY ? 0 : ex2(e.x - M_));     // a NaN sum stays one: scores of NaN move no maximum
        }
        float acc[GROUPS * 4];
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) {
            float4 a = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                const float *src = reinterpret_cast<const float *>(smem + (i * F::STAGES + stage) * F::STAGE) + row * D;
                const float4 b = *reinterpret_cast<const float4 *>(src + (((j * TPR + lanec) * 4) ^ ((row >> 1 & 3) * 8)));
                a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w;
            }
            acc[j * 4] = a.x, acc[j * 4 + 1] = a.y, acc[j * 4 + 2] = a.z, acc[j * 4 + 3] = a.w;
        }
        bool write = whole;
        if (!whole) {
            // this worker's part, and whoever brings the last part of the tile joins them
            const uint32_t w0 = (uint32_t)quotient((tile0 + 1) * workers - 1, total);
            const uint32_t w1 = (uint32_t)quotient((tile0 + get.n_units) * workers - 1, total);
            auto slot = [&](uint32_t i) { return i == w0 ? 2 * i + 1 : 2 * i; };
            float *part_o = ws.part, *part_ml = ws.part + (uint64_t)2 * ws.workers * F::ROWS * D;
            float4 *po = reinterpret_cast<float4 *>(part_o + ((uint64_t)slot(w) * F::ROWS + row) * D);
#pragma unroll
            for (int j = 0; j < GROUPS; ++j) po[j * TPR + lanec] = make_float4(acc[j * 4], acc[j * 4 + 1], acc[j * 4 + 2], acc[j * 4 + 3]);
            if (lanec == 0) reinterpret_cast<float2 *>(part_ml)[slot(w) * F::ROWS + row] = make_float2(M_, L);
            __syncthreads();
            if (threadIdx.x == 0) {
                const uint32_t old = arrive_gpu(ws.count + w0);
                if (old == w1 - w0) ws.count[w0] = 0;          // ready for the next call
                plan[0] = old == w1 - w0;
            }
            __syncthreads();
            write = plan[0];
            if (write) {
                // in worker order, a running maximum along, the loads of several parts in flight at once
                const float2 *parts_ml = reinterpret_cast<const float2 *>(part_ml);
                M_ = -INFINITY;
                L = 0;
#pragma unroll
                for (int j = 0; j < GROUPS * 4; ++j) acc[j] = 0;
                constexpr int IN_FLIGHT = C8 ? DEEP_8 : DEEP;
#pragma unroll IN_FLIGHT
                for (uint32_t i = w0; i <= w1; ++i) {
                    const float2 e = __ldcg(parts_ml + slot(i) * F::ROWS + row);
                    const float4 *src = reinterpret_cast<const float4 *>(part_o + ((uint64_t)slot(i) * F::ROWS + row) * D);
                    float4 b[GROUPS];
#pragma unroll
                    for (int j = 0; j < GROUPS; ++j) b[j] = __ldcg(src + j * TPR + lanec);
                    const float m2 = fmaxf(M_, e.x);
                    const float was = m2 == -INFINITY ? 0 : ex2(M_ - m2), f = m2 == -INFINITY ? 0 : ex2(e.x - m2);
                    M_ = m2;
                    L = L * was + e.y * f;
#pragma unroll
                    for (int j = 0; j < GROUPS; ++j) {
                        acc[j * 4] = acc[j * 4] * was + b[j].x * f, acc[j * 4 + 1] = acc[j * 4 + 1] * was + b[j].y * f;
                        acc[j * 4 + 2] = acc[j * 4 + 2] * was + b[j].z * f, acc[j * 4 + 3] = acc[j * 4 + 3] * was + b[j].w * f;
                    }
                }
            }
        }
        if (write && row0 + row < n_rows) {
            const uint32_t i = token_of(row0 + row), qh = h * p.group + (row0 + row - i * p.group);
            const uint64_t tok = get.v.q0 + i;
            const float inv = L == 0 ? 0.0f : 1.0f / L;
            T *out = (T *)p.out + tok * p.out_stride + (uint64_t)qh * D;
#pragma unroll
            for (int j = 0; j < GROUPS; ++j)
                *reinterpret_cast<uint2 *>(out + (j * TPR + lanec) * 4) =
                    make_uint2(pack2(acc[j * 4] * inv, acc[j * 4 + 1] * inv, T()), pack2(acc[j * 4 + 2] * inv, acc[j * 4 + 3] * inv, T()));
            if (p.lse && lanec == 0)
                p.lse[tok * p.n_q_heads + qh] = L == 0 ? -INFINITY : (M_ - F::OFF + log2f(L)) * 0.6931471805599453f;
        }
        __syncthreads();                     // the stage and the small arrays may be written again
        stage = stage + 1 == F::STAGES ? 0 : stage + 1;
        if (x < x1) advance(p, F::ROWS, F::UNIT, get);
    }
    cp_wait<0>();
}

template <typename T, bool C8, int D, int NB, bool WIN>
cudaError_t launch_few(const AttendParams &p, Workspace ws, int sms, cudaStream_t st) {
    using F = Few<T, C8, D, NB>;
    ws.workers = sms * F::WORKERS_PER_SM;
    if constexpr (WIN) return launch_behind(attend_few_kernel<T, C8, D, NB, WIN>, ws.workers, WARPS * 32, F::SMEM, st, p, ws);
    else return launch_plain(attend_few_kernel<T, C8, D, NB, WIN>, ws.workers, WARPS * 32, F::SMEM, st, p, ws);
}

template <typename T, bool C8, int D, int NB, bool WIN>
cudaError_t setup_few() {
    return cudaFuncSetAttribute(attend_few_kernel<T, C8, D, NB, WIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, Few<T, C8, D, NB>::SMEM);
}

// f(type, 8-bit, head_dim, row blocks, window) for one or for every instance
template <typename F>
cudaError_t pick(bool bf, bool c8, bool wide, bool two, bool window, F f) {
    auto win = [&](auto t, auto c, auto d, auto n) { return window ? f(t, c, d, n, std::true_type()) : f(t, c, d, n, std::false_type()); };
    auto nb = [&](auto t, auto c, auto d) {
        return two ? win(t, c, d, std::integral_constant<int, 2>()) : win(t, c, d, std::integral_constant<int, 1>());
    };
    auto dim = [&](auto t, auto c) {
        return wide ? nb(t, c, std::integral_constant<int, 128>()) : nb(t, c, std::integral_constant<int, 64>());
    };
    auto cache = [&](auto t) { return c8 ? dim(t, std::true_type()) : dim(t, std::false_type()); };
    return bf ? cache(__nv_bfloat16()) : cache(__half());
}

}  // namespace

cudaError_t few_setup() {
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < 32 && e == cudaSuccess; ++i)
        e = pick(i & 1, i & 2, i & 4, i & 8, i & 16, [](auto t, auto c, auto d, auto nb, auto w) { return setup_few<decltype(t), c.value, d.value, nb.value, w.value>(); });
    return e;
}

cudaError_t few_launch(const AttendParams &p, const Workspace &ws, int sms, bool c8, bool bf, cudaStream_t st) {
    // one block of 8 rows where a step's tokens and the query heads of a KV head fit
    const bool two = (uint64_t)p.step.max_new * p.group > 8;
    return pick(bf, c8, p.pool.head_dim == 128, two, p.window != 0, [&](auto t, auto c, auto d, auto nb, auto w) {
        return launch_few<decltype(t), c.value, d.value, nb.value, w.value>(p, ws, sms, st);
    });
}

// of the instance with the most
uint32_t few_workers(int sms) { return (uint32_t)sms * 4; }
size_t few_part_bytes(int sms) { return (size_t)2 * sms * 4 * 8 * (128 + 2) * sizeof(float); }

}  // namespace tutti
