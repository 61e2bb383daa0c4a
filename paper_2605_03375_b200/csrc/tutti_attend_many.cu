// Attention of many rows per sequence (a prompt chunk behind a restored prefix, a speculative
// step): both products on the 5th-generation tensor cores.
//
// A *tile* is 256 rows of one sequence and KV head, two halves of 128 rows (the M of one
// tcgen05.mma), against keys in units of 128.  As in the few-row kernel all units of all tiles
// are dealt out evenly over the SMs, one worker (CTA) each, and a tile that several workers share
// is joined by the last of them; a causal tile's units are counted in closed form (floor_sum), so
// a captured graph follows lengths that change.
//
// Roles of a worker's 16 warps:
//   0-3, 4-7  softmax of half 0 / half 1: a thread owns a row, reads its scores from TMEM, writes
//             its probabilities back over them (16 bits), rescales the output when the running
//             maximum has grown by more than 2^8, and writes the row out at the end;
//   8         issues the matrix instructions: S = Q K^T (both operands in shared memory),
//             O += P V (P from TMEM, over the scores it came from).  16-bit caches: a unit is one step of
//             128 keys; a half's next scores wait for its P V, which waits for its softmax, while the other
//             half has the tensor cores.  8-bit caches: two steps of 64 keys, each with its own columns of
//             scores, so that a step's scores are ready before the softmax of the step before it has ended.
//             An instruction of 128 x 64 x 16 reads 6 KB of shared memory in the time of 4 KB, which makes
//             Q K^T 1.5 times as long: it costs a 16-bit cache more than the waiting (318 against 278 us),
//             and an 8-bit one, where the widening warps are the bound, less (360 -> 311);
//   9-11      bring the queries of the next tile; 9 also walks over the worker's tiles and publishes them (Share);
//   12-15     gather keys and values through the block table into a ring of four 128-row tiles
//             in the 128-byte swizzle (K: K-major B operand, V: the same bytes read as an
//             MN-major B operand): one tensor copy per block and 128 bytes of its rows, or, where a
//             sequence ends inside the unit, a block is missing or blocks do not tile 64 rows, row
//             by row with zeros in place of what is not there.  Two groups of two warps take the
//             units in turn, so a group waits for its own loads while the other's are in flight.
//             8-bit codes are widened to 16 bits (code * scale; f16 in units of a power of two for the 64 keys of
//             a step, which the softmax warps undo): keys where they landed, values out of a buffer of their
//             own, so that they are fetched before the place they go to is free.
// Bound: the tensor cores (2 x 128 x 128 x D multiply-adds a half and unit: 2048 clocks a unit for D = 128)
// and, as close, the 2 x 128 x 128 exponentials on 16 lanes a clock; in a long loop the power limit
// (1550 MHz at 1000 W).  What is reached: 3500-4000 clocks a unit, set by the chain scores -> softmax -> P V
// -> next scores of a half.  A tile's start and end cost about two units more: they are code that runs once a tile, and the
// roles' code together does not fit the instruction cache, so that what is rare is kept small (masks as bits, outputs in
// pieces, one walk over the tiles; 2048 tokens without a prefix 97 -> 61 us).
// On a B200 (1694 TFLOP/s in short, 1395 in long runs of the library's product), the kernel
// alone, 32 heads: 2048 new tokens over 32768, bf16, 1133 us = 1000 TFLOP/s; 1801 over 2 x 8192 235-270 us = 930-1070
// (264 us among other calls); 8-bit, fp16, 4 ragged chunks over 2000-9000 232 us = 810, bf16 291 us (the widening of the codes
// and shared memory); 64-wide heads 1801 over 2 x 8192 198 us = 640.
//
// Under a window (WIN) a tile's keys are the sequence's first tokens and the ones from its first row's window on, laid end to end
// (WindowRows), so that 4 first tokens do not cost a unit of 128 and the window need not begin with one; with units of the sequence's
// own keys, those in between left out, 8-bit chunks under a window of 1024 took 86 us instead of 74, 8192 rows under one of 128 95
// instead of 78.  8192 tokens without a prefix, 4 first tokens, bf16: window 128 78 us, 1024 185 us = 700 TFLOP/s,
// 4096 over 24576 505-555 us = 990-1080; 8-bit, fp16, 4 chunks of 300-700 under a window of 1024 74 us, bf16 82 us.
#include <cstring>
#include <type_traits>

#include "tutti_attend.h"

namespace tutti {

namespace {

constexpr int HALF_ROWS = 128;
constexpr int TILE_ROWS = 256;
constexpr int BN = 128;                 // keys of a unit
constexpr int RING = 4;                 // K and V tiles in flight
constexpr uint32_t SNAP = 3;            // units
constexpr int MIN_UNITS = 4;            // of a worker that takes a part of a tile
constexpr int THREADS = 512;
constexpr int MMA_WARP = 8, Q_WARP = 9, Q_WARPS = 3, KV_WARP = 12, KV_WARPS = 2;      // KV_WARPS: of a group
constexpr uint32_t ATOM = BN * 128;     // 128 rows of 128 bytes
constexpr int SUB_16 = 128, SUB_8 = 64;  // keys of a step, by the cache's bits
constexpr int REGS_16 = 192, REGS_8 = 160;  // of a softmax thread; the other half of the threads has 256 less these
constexpr float GROW = 8.0f;            // log2 of how far probabilities may exceed 1
// Exponents of the units of f16 operands (see unit_of).  Keys: any.  Values: 2 at least, the unit of nearly every
// cache (f16 rows give scales of 2^8 at most), so that the output's unit changes only for larger ones; what is
// lost below is 2^-24, the smallest step that an f16 output has.  2^64 at most: parts are joined by 32-bit weights.
constexpr int UNIT_LEAST_K = -120, UNIT_MOST_K = 120, UNIT_LEAST_V = 1, UNIT_MOST_V = 64;
constexpr long long WAIT_CLOCKS = 3000000000ll;   // about 1.5 s: a wait that takes longer is given up

// sum over i in [0, n) of floor((a i + b) / m)  (a, b >= 0, m > 0): whole parts of a / m and b / m in closed form, then
// the reciprocity of such sums (Graham, Knuth and Patashnik, Concrete Mathematics, section 3.5), which exchanges a
// and m as Euclid's algorithm does.
template <typename U>
__host__ __device__ inline uint64_t floor_sum_in(U n, U m, U a, U b) {
    uint64_t ans = 0;
    while (n) {
        if (a >= m) {
            const U q = a / m;
            ans += (uint64_t)n * (n - 1) / 2 * q;
            a -= q * m;
        }
        if (b >= m) {
            const U q = b / m;
            ans += (uint64_t)n * q;
            b -= q * m;
        }
        const U y = a * n + b;
        if (y < m) break;
        n = y / m;
        b = y - n * m;
        const U t = m;
        m = a;
        a = t;
    }
    return ans;
}
// In 32 bits where all of it fits (a n + b bounds every value on the way): their division is much faster.
__host__ __device__ inline uint64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b) {
    if (n < (1u << 20) && a < (1u << 11) && m < (1u << 31) && a * n + b < (1ull << 31))
        return floor_sum_in<uint32_t>((uint32_t)n, (uint32_t)m, (uint32_t)a, (uint32_t)b);
    return floor_sum_in<uint64_t>(n, m, a, b);
}

// The tiles of one sequence and head.
struct Rows {
    uint32_t n_rows, n_tiles, group, ctx;
    uint32_t group_mul, group_shift;    // row / group = row * group_mul >> group_shift
    int64_t first;                      // position of the first new token
    __host__ __device__ uint32_t token_of(uint32_t row) const { return (uint32_t)((uint64_t)row * group_mul >> group_shift); }
    // units of tile q: up to the key of its last row
    __host__ __device__ uint32_t units(uint32_t q) const {
        if (first < 0 || ctx == 0) return ctx ? (ctx + BN - 1) / BN : 1;     // padding rows: every tile sees all
        const uint32_t end = q + 1 < n_tiles ? (q + 1) * TILE_ROWS : n_rows;
        return ((uint32_t)first + token_of(end - 1)) / BN + 1;
    }
    // units of tiles [0, q)
    __host__ __device__ uint64_t before(uint32_t q) const {
        if (q == 0) return 0;
        if (first < 0 || ctx == 0) return (uint64_t)q * units(0);
        // floor((first + floor(x / group)) / BN) = floor((first group + x) / (BN group)), x = 256 (i + 1) - 1
        const uint32_t full = q == n_tiles ? q - 1 : q;
        const uint64_t sum = full + floor_sum(full, (uint64_t)BN * group, TILE_ROWS, (uint64_t)first * group + TILE_ROWS - 1);
        return q == n_tiles ? sum + units(q - 1) : sum;
    }
};

// The same under a window.  From tile q0 on, where it saves a unit at least, a tile's keys are laid end to end without the ones
// that none of its rows sees: the first `front` of the sequence, then the ones from its first row's window on (a
// multiple of `grain`).  All such tiles have `per` units, what the longest of them needs, so that sums over tiles stay closed forms.
struct WindowRows : Rows {
    uint32_t q0, per, front, grain;
    int64_t start;                      // first key of the first row's window
    // Key number v of tile q is key v of the sequence below `front`, and key v + shift(q) from there on; 0: of a tile in front of q0.
    __host__ __device__ uint32_t shift(uint32_t q) const { return q < q0 ? 0 : (uint32_t)(start + token_of(q * TILE_ROWS)) / grain * grain - front; }
    __host__ __device__ uint32_t units(uint32_t q) const { return q < q0 ? Rows::units(q) : per; }
    __host__ __device__ uint64_t before(uint32_t q) const { return q <= q0 ? Rows::before(q) : Rows::before(q0) + (uint64_t)(q - q0) * per; }
};
template <bool WIN> struct RowsOf { typedef Rows type; };
template <> struct RowsOf<true> { typedef WindowRows type; };

__host__ __device__ inline void rows_of(const SeqView &v, const AttendParams &p, Rows &r) {
    r.n_rows = v.n_new * p.group;
    r.n_tiles = (r.n_rows + TILE_ROWS - 1) / TILE_ROWS;
    r.group = p.group;
    r.group_mul = p.group_mul;
    r.group_shift = p.group_shift;
    r.ctx = v.ctx;
    r.first = (int64_t)v.ctx - v.n_new;
}
__host__ __device__ inline void rows_of(const SeqView &v, const AttendParams &p, WindowRows &r) {
    rows_of(v, p, static_cast<Rows &>(r));
    r.front = p.front;
    r.grain = p.grain;
    r.start = p.window_start(r.first);
    // the first tile whose window begins a unit or more behind `front`: floor(256 q / group) tokens behind the first row's; padding rows: none
    const int64_t x = (int64_t)p.front + BN - r.start;
    const uint64_t q0 = x > 0 ? ((uint64_t)x * p.group + TILE_ROWS - 1) / TILE_ROWS : 0;
    r.q0 = r.first < 0 || q0 > 0xffffffffu ? 0xffffffffu : (uint32_t)q0;
    // tokens of a tile at most, and how far its window's start may lie behind a multiple of grain
    const uint32_t tokens = TILE_ROWS % p.group ? (TILE_ROWS - 2 + p.group) / p.group + 1 : TILE_ROWS / p.group;
    const uint32_t slack = TILE_ROWS % p.group || tokens % p.grain || r.start < 0 ? p.grain - 1 : (uint32_t)(r.start % p.grain);
    r.per = (uint32_t)(((uint64_t)p.front + tokens + p.window - 1 + slack + BN - 1) / BN);
}

// Where a cut at unit u of a tile of n units goes: to its start below low(n), behind it from n -
// high(n) on (a tile of 2 SNAP units or less is never cut).
__host__ __device__ inline uint32_t snap_low(uint32_t n) { return n <= 2 * SNAP ? (n + 1) / 2 : SNAP; }
__host__ __device__ inline uint32_t snap_high(uint32_t n) { return n <= 2 * SNAP ? n / 2 : SNAP; }
__host__ __device__ inline uint32_t snapped(uint32_t u, uint32_t n) { return u < snap_low(n) ? 0 : u >= n - snap_high(n) ? n : u; }
// Unit at which worker w's share starts, before it is moved.
__host__ __device__ inline unsigned long long cut_of(unsigned long long w, unsigned long long workers, unsigned long long total) {
    return quotient(w * total, workers);
}
// The first and the last worker that have a part of a tile of n units that starts at unit tile0: those whose
// first and last cut before the tile's end lie in front of it and inside.
__host__ __device__ inline void holders(unsigned long long tile0, uint32_t n, unsigned long long workers, unsigned long long total, uint32_t &w0, uint32_t &w1) {
    w0 = (uint32_t)quotient((tile0 + snap_low(n)) * workers - 1, total);
    w1 = (uint32_t)quotient((tile0 + n - snap_high(n)) * workers - 1, total);
}

template <bool WIN>
struct Tile {
    uint32_t s, h, q, u, n_units;
    SeqView v;
    typename RowsOf<WIN>::type r;
};

// The sequence of a cut: units of one of its heads, units in front of the cut.
template <bool WIN>
struct Found {
    Tile<WIN> t;
    unsigned long long head, in_seq;
};

// What is added to a key's number in the tile, from p.front on.
template <bool WIN>
__device__ inline uint32_t shift_of(const Tile<WIN> &t) {
    if constexpr (WIN) return t.r.shift(t.q);
    else return 0;
}

template <bool WIN>
__device__ inline int tile_seq(const AttendParams &p, uint32_t s, Tile<WIN> &t) {
    t.s = s;
    const int code = seq_view(p.step, p.pool.block_tokens, s, t.v);
    if (code != TUTTI_OK) t.v.n_new = t.v.ctx = 0;
    rows_of(t.v, p, t.r);
    return code;
}

template <bool WIN>
__device__ inline void next_tile(const AttendParams &p, Tile<WIN> &t) {
    t.u = 0;
    if (++t.q == t.r.n_tiles) {
        t.q = 0;
        if (++t.h == p.pool.n_kv_heads) {
            t.h = 0;
            do {
                if (t.s + 1 >= p.step.n_seq) return;          // behind the last tile: not used
                tile_seq(p, t.s + 1, t);
            } while (t.r.n_tiles == 0);
        }
    }
    t.n_units = t.r.units(t.q);
}

// ---- instructions ----

__device__ inline void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ inline void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ inline bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
// Bounded: false once this wait, or any other of the CTA, has been given up.
__device__ inline bool mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *dead) {
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
    while (!mbar_try(bar, parity)) {
        if (*dead) return false;
        if (clock64() - t0 > WAIT_CLOCKS) {
            *dead = 1;
            return false;
        }
    }
    return true;
}
__device__ inline void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ inline void tile_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t c0, int32_t c1, int32_t c2, int32_t c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ inline void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ inline void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ inline void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ inline void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
template <int R> __device__ __forceinline__ void setmaxnreg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R> __device__ __forceinline__ void setmaxnreg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }
__device__ inline void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ inline void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ inline void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc) : "memory");
}
__device__ inline void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc) : "memory");
}

#define O4(a, i) "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3])
#define I4(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3])
__device__ inline void tc_ld32(uint32_t *r, uint32_t a) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : O4(r, 0), O4(r, 4), O4(r, 8), O4(r, 12), O4(r, 16), O4(r, 20), O4(r, 24), O4(r, 28) : "r"(a));
}
#define P4(a, i) "+r"(a[i]), "+r"(a[i + 1]), "+r"(a[i + 2]), "+r"(a[i + 3])
// Behind tc_wait_ld: no use of the loaded registers may be moved in front of the wait.
__device__ inline void tc_loaded(uint32_t *r) {
    asm volatile("" : P4(r, 0), P4(r, 4), P4(r, 8), P4(r, 12), P4(r, 16), P4(r, 20), P4(r, 24), P4(r, 28));
}
__device__ inline void tc_st16(const uint32_t *r, uint32_t a) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::I4(r, 0), I4(r, 4), I4(r, 8), I4(r, 12), "r"(a) : "memory");
}

__device__ inline void tc_ld16(uint32_t *r, uint32_t a) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : O4(r, 0), O4(r, 4), O4(r, 8), O4(r, 12) : "r"(a));
}

__device__ inline bool elect() {
    uint32_t x;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(x));
    return x;
}

// ---- arithmetic on pairs ----
typedef unsigned long long f2;
__device__ inline f2 pair(float a, float b) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ inline void unpair(f2 x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ inline f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ inline f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ inline float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Shared-memory operand in the 128-byte swizzle: start, offset between 64-element groups of an
// MN-major operand (not used by a K-major one), 1024 bytes from one group of 8 rows to the next.
__device__ inline uint64_t operand(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(ATOM >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// Four codes as two pairs of 16-bit elements, not yet at their scale.  f16: the values, in order.
__device__ inline uint2 spread(uint32_t w, __half) {
    uint2 r;
    codes4(w, r.x, r.y);
    return r;
}
// bf16: codes 0, 2 and 1, 3 (the queries are brought in the same order and the outputs leave in it),
// the magnitude's 7 bits moved to where they are the value times 2^-120, subnormal codes included.
// NaN codes become 480 * 2^-120, the largest magnitude there is: `top` collects the magnitudes.
__device__ inline uint2 spread(uint32_t w, __nv_bfloat16, uint32_t &top) {
    const uint32_t even = (w << 4) & 0x07f007f0u, odd = (w >> 4) & 0x07f007f0u;
    top = __vmaxu2(__vmaxu2(top, even), odd);
    return make_uint2(even | ((w << 8) & 0x80008000u), odd | (w & 0x80008000u));
}
__device__ inline uint2 spread(uint32_t w, __half, uint32_t &) { return spread(w, __half()); }
template <typename P>
__host__ __device__ inline uint32_t word(const P &x) {
    uint32_t w;
    memcpy(&w, &x, 4);
    return w;
}
template <typename P>
__host__ __device__ inline P pair_of(uint32_t w) {
    P x;
    memcpy((void *)&x, &w, 4);
    return x;
}
__host__ __device__ inline uint32_t twice(float x, __half) { return word(__float2half2_rn(x)); }
__host__ __device__ inline uint32_t twice(float x, __nv_bfloat16) { return word(__float2bfloat162_rn(x)); }
__host__ __device__ inline uint32_t times(uint32_t x, uint32_t s, __half) { return word(__hmul2(pair_of<__half2>(x), pair_of<__half2>(s))); }
__host__ __device__ inline uint32_t times(uint32_t x, uint32_t s, __nv_bfloat16) {
    return word(__hmul2(pair_of<__nv_bfloat162>(x), pair_of<__nv_bfloat162>(s)));
}
// f16 operands of an 8-bit cache are kept in units of a power of two, one for the keys and one for the values of
// a step's 64 rows: the exponent that brings their largest scale (its bits) to 2^7 at most, so that no code
// times scale passes 448 * 2^7, between `least` and `most`.
__host__ __device__ inline int unit_of(uint32_t top, int least, int most) {
    const int e = (int)((top + 0x7fffffu) >> 23) - 127 - 7;        // the power of two at or above it
    return e < least ? least : e > most ? most : e;
}
__host__ __device__ inline float pow2(int e) {                     // -126 <= e <= 127
    const uint32_t w = (uint32_t)(e + 127) << 23;
    float x;
    memcpy(&x, &w, 4);
    return x;
}
// A scale as the two factors that finish spread(), each rounded to the type (powers of two are
// exact) and twice in a register; true if the second is not 1.  f16 (a scale in its unit, 2^7 at most): one below
// the normal range is brought in 2^14 times too large, which is below 1, so the code times it stays below 448
// and the second factor rounds once, into the subnormal range where the product lies there.
__host__ __device__ inline bool factors(float s, uint32_t &f1, uint32_t &f2, __half) {
    const bool low = s != 0 && fabsf(s) < 0x1p-14f;
    f1 = twice(low ? s * 0x1p14f : s, __half());
    f2 = twice(low ? 0x1p-14f : 1.0f, __half());
    return low;
}
__host__ __device__ inline bool factors(float s, uint32_t &f1, uint32_t &f2, __nv_bfloat16) {
    const bool high = fabsf(s) >= 128.0f;                                     // 2^120 * s would overflow
    f1 = twice(high ? 1.329227995784916e+36f : 1.329227995784916e+36f * s, __nv_bfloat16());
    f2 = twice(high ? s : 1.0f, __nv_bfloat16());
    return high;
}

// The units [u, u + n) of a tile of n_units that a worker has: published by the warps that bring the queries, so that the
// walk over tiles stands in the code of fewer roles.  The products' warp has read a share before the queries of the next are
// brought; the softmax warps say when they have.
constexpr uint32_t SHARES = 4;
struct Share {
    uint32_t n, u, n_units, shift;      // shift: see WindowRows
    uint32_t q, h, q0, n_rows;          // tile of the head, KV head, first row of the sequence in the step, rows of a head
    int64_t first;                      // position of the first new token
};

template <typename T, bool C8, int D>
struct Many {
    static constexpr int SUB = C8 ? SUB_8 : SUB_16, STEPS = BN / SUB;
    static constexpr int SOFT_REGS = C8 ? REGS_8 : REGS_16;
    static constexpr uint32_t KV = ATOM * (D / 64);         // bytes of a 128-row tile
    static constexpr uint32_t OFF_RING = 2 * KV;            // behind the two halves of Q
    static constexpr uint32_t OFF_RAW = OFF_RING + RING * KV;          // 8-bit: codes of a group's values
    static constexpr uint32_t OFF_BAR = OFF_RAW + (C8 ? 2 * ATOM : 0);
    static constexpr uint32_t OFF_EXISTS = OFF_BAR + 352;   // [8 units][4]: keys that exist
    static constexpr bool UNITS = C8 && std::is_same<T, __half>::value;
    static constexpr uint32_t OFF_UNITS = OFF_EXISTS + 128; // [8 units][2 steps]: exponents of keys' and values' units
    static constexpr uint32_t OFF_MISC = OFF_UNITS + (UNITS ? 128 : 0);
    static constexpr uint32_t OFF_TILE = OFF_MISC + 320;
    static constexpr uint32_t OFF_SHARE = OFF_TILE + 256;   // [SHARES] what the worker has of its tiles
    static constexpr uint32_t SMEM = OFF_SHARE + SHARES * sizeof(Share) + 1024;     // 1024: alignment of the dynamic part
    // f16 probabilities are kept 2^6 times too large (at most 2^14): full precision down to 2^-20
    static constexpr float OFF = std::is_same<T, __half>::value ? 6.0f : 0.0f;
    // whether widened codes keep their order
    static constexpr bool ORDERED = !C8 || std::is_same<T, __half>::value;
    // byte offset of 16-byte chunk `ch` of row `row` in a tile
    __device__ static uint32_t place(uint32_t row, uint32_t ch) {
        return (ch >> 3) * ATOM + row * 128 + (((ch ^ row) & 7) << 4);
    }
};

template <typename T, bool C8, int D, bool WIN>
__global__ void __launch_bounds__(THREADS, 1) attend_many_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ PoolMaps maps, const Workspace ws) {
    using C = Many<T, C8, D>;
    constexpr int SUB = C::SUB, STEPS = C::STEPS;
    if constexpr (WIN) asm volatile("griddepcontrol.wait;" ::: "memory");
    extern __shared__ unsigned char raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    unsigned char *sm = raw + (base - smem_addr(raw));
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    uint32_t *misc = reinterpret_cast<uint32_t *>(sm + C::OFF_MISC);
    uint32_t *exists = reinterpret_cast<uint32_t *>(sm + C::OFF_EXISTS);
    Found<WIN> *found = reinterpret_cast<Found<WIN> *>(sm + C::OFF_TILE);
    static_assert(2 * sizeof(Found<WIN>) <= 256, "two of them lie in front of the end");
    int2 *units = reinterpret_cast<int2 *>(sm + C::OFF_UNITS);
    volatile uint32_t *dead = misc + 72;
    const uint32_t bars = base + C::OFF_BAR;
    const uint32_t full = bars, empty = bars + 32, q_full = bars + 64, q_empty = bars + 72, o_full = bars + 80, o_empty = bars + 96,
                   joined = bars + 112, drain = bars + 128, raw_full = bars + 136, s_full = bars + 200, p_full = bars + 232, o_done = bars + 264, share_full = bars + 280, share_free = bars + 312;
    Share *shares = reinterpret_cast<Share *>(sm + C::OFF_SHARE);

    // ---- this worker's share ----
    unsigned long long *sums = reinterpret_cast<unsigned long long *>(misc);
    const uint32_t per = (p.step.n_seq + THREADS - 1) / THREADS;
    const uint32_t s_lo = threadIdx.x * per, s_hi = min(s_lo + per, p.step.n_seq);
    unsigned long long mine = 0;
    uint32_t my_tiles = 0;
    Found<WIN> own;                                // the thread's last sequence (its only one, mostly)
    own.t.s = ~0u;
    auto look = [&](uint32_t s) {
        const int code = tile_seq(p, s, own.t);
        own.head = own.t.r.before(own.t.r.n_tiles);
        return code;
    };
    for (uint32_t s = s_lo; s < s_hi; ++s) {
        const int code = look(s);
        if (code != TUTTI_OK && blockIdx.x == 0) report(p.step, code);
        mine += own.head * p.pool.n_kv_heads;
        my_tiles += own.t.r.n_tiles * p.pool.n_kv_heads;
    }
    unsigned long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    my_tiles = __reduce_add_sync(0xffffffffu, my_tiles);
    if (lane == 31) sums[warp] = incl, misc[48 + warp] = my_tiles;
    __syncthreads();
    uint32_t tiles = 0;
    unsigned long long total = 0, start = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i < (int)warp) start += sums[i];
        total += sums[i];
        tiles += misc[48 + i];
    }
    start += incl - mine;
    unsigned long long workers = (total + MIN_UNITS - 1) / MIN_UNITS;
    if (workers < tiles) workers = tiles;
    if (workers > ws.workers) workers = ws.workers;
    if (workers > total) workers = total;
    const uint32_t w = blockIdx.x;
    if (w >= workers) return;
    // The share [x0, x1): cuts at multiples of total / workers, moved to a tile's end where one is near.
    // Threads find the sequences of both cuts, warps 0 and 1 the tiles.
    const unsigned long long cut[2] = {cut_of(w, workers, total), cut_of(w + 1, workers, total)};
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (cut[i] >= start && cut[i] < start + mine) {
            unsigned long long at = start;
            for (uint32_t s = s_lo; s < s_hi; ++s) {
                if (s != own.t.s) look(s);
                const unsigned long long n = own.head * p.pool.n_kv_heads;
                if (cut[i] < at + n) {
                    own.in_seq = cut[i] - at;
                    found[i] = own;
                    break;
                }
                at += n;
            }
        }
    if (threadIdx.x == 0) {
        for (int i = 0; i < RING; ++i) {
            mbar_init(full + 8 * i, KV_WARPS);
            mbar_init(empty + 8 * i, 1);
        }
        mbar_init(q_full, Q_WARPS);
        mbar_init(q_empty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(o_full + 8 * i, 1);
            mbar_init(o_done + 8 * i, 1);
            mbar_init(o_empty + 8 * i, 4);
            mbar_init(joined + 8 * i, 4);
        }
        for (int i = 0; i < 4; ++i) {               // half x step of a unit
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 4);
        }
        mbar_init(drain, 1);
        for (uint32_t i = 0; i < SHARES; ++i) {
            mbar_init(share_full + 8 * i, 1);
            mbar_init(share_free + 8 * i, MMA_WARP);        // the softmax warps
        }
        for (int i = 0; i < 2 * RING; ++i) mbar_init(raw_full + 8 * i, 1);
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(base + C::OFF_MISC + 73 * 4) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_before();
    }
    __syncthreads();
    tc_after();
    const uint32_t tmem = misc[73];
    if (warp < 2) {
        unsigned long long x = cut[warp];
        Tile<WIN> f;
        f.s = f.h = f.q = f.u = f.n_units = 0;
        if (x < total) {
            f = found[warp].t;
            const auto r = f.r;
            const unsigned long long in_seq = found[warp].in_seq, head = found[warp].head;
            f.h = (uint32_t)quotient(in_seq, head);
            const unsigned long long rest = in_seq - f.h * head;
            unsigned long long at = 0;                  // units in front of tile `lo`
            uint32_t lo = 0, len = r.n_tiles;           // last tile that starts at or before `rest`, 32 probes a round
            while (len > 1) {
                const uint32_t step = (len + 31) / 32;
                const unsigned long long mine = lane * step < len ? r.before(lo + lane * step) : ~0ull;
                const uint32_t last = 31 - __clz(__ballot_sync(0xffffffffu, mine <= rest) | 1u);
                at = __shfl_sync(0xffffffffu, mine, last);
                lo += last * step;
                len = min(len - last * step, step);
            }
            f.q = lo;
            f.u = (uint32_t)(rest - at);
            f.n_units = r.units(lo);
            const uint32_t u = snapped(f.u, f.n_units);
            x = x - f.u + u;
            f.u = u;
            if (u == f.n_units && x < total) next_tile(p, f);
        }
        __syncwarp();
        if (lane == 0) {
            sums[22 + warp] = x;
            if (warp == 0) found[0].t = f;
        }
    }
    __syncthreads();
    const unsigned long long x0 = sums[22], x1 = sums[23];
    Tile<WIN> t = found[0].t;
    // scores (and probabilities over them) of a half and step, then the halves' outputs
    auto S = [&](int i, int u) { return tmem + i * 128 + u * SUB; };
    auto O = [&](int i) { return tmem + 256 + i * D; };

    // Registers: 512 x 128 at launch = 256 x 160 + 256 x 96; a softmax thread holds 64 scores.
    if (warp >= MMA_WARP) {
        setmaxnreg_dec<256 - C::SOFT_REGS>();
        if (warp >= KV_WARP) {
        // =================================== keys and values ===================================
        const uint32_t group = (warp - KV_WARP) / KV_WARPS, half = (warp - KV_WARP) % KV_WARPS;     // rows [64 half, 64 half + 64)
        constexpr int RB = D * (C8 ? 1 : 2);            // bytes of a row in the pool
        constexpr int CH = RB / 16, RPI = 32 / CH;      // its 16-byte chunks; rows a warp takes at once
        const uint32_t ch = lane % CH, sub = lane / CH;
        const uint32_t slot0 = C::OFF_RING + 2 * group * C::KV;           // K's place; V's is the next
        // Where the rows of the pool land: 16-bit ones in their places, 8-bit keys in the upper half
        // of theirs, 8-bit values in the group's buffer (128 bytes from row to row, swizzled alike).
        const uint32_t land[2] = {slot0 + (C8 && D == 128 ? ATOM : 0), C8 ? C::OFF_RAW + group * ATOM : slot0 + C::KV};
        const uint32_t bs = p.pool.block_tokens, box_rows = min(bs, 64u), boxes = 64 / box_rows;
        const uint32_t my_box = lane % boxes, my_part = lane / boxes;    // of a lane's tensor copy
        uint32_t raw_phase = 0;
        bool ok = true;
        unsigned long long fx = x0;
        auto step_unit = [&]() {
            ++fx;
            if (fx < x1 && ++t.u == t.n_units) next_tile(p, t);
        };
        // The next unit: block ids of rows lane and lane + 32 (locate), then what follows from them.
        int32_t id[2];
        uint32_t key0 = 0, head = 0, ctx = 0, start = 0, shift = 0;
        auto key_of = [&](uint32_t v) { return WIN && v >= p.front ? v + shift : v; };
        auto in_sight = [&](uint32_t key) { return key < ctx && (!WIN || key < p.sinks || key >= start); };
        int64_t off[2];
        float ks[2], vs[2];
        uint32_t missing[2];
        bool tiled = false;
        auto locate = [&]() {
            key0 = t.u * BN + half * 64;
            shift = shift_of(t);
            head = t.h;
            ctx = fx < x1 ? t.v.ctx : 0;
            if constexpr (WIN) {                        // of the sequence: no row sees a key in front of its first row's window
                const int64_t x = p.window_start(t.r.first);
                start = x > 0 ? (uint32_t)x : 0;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t key = key_of(key0 + i * 32 + lane);
                id[i] = in_sight(key) ? __ldg(p.step.block_ids + t.v.b0 + p.pool.block_of(key)) : -1;
            }
        };
        auto resolve = [&]() {
            tiled = maps.valid;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t key = key_of(key0 + i * 32 + lane);
                const bool there = (uint32_t)id[i] < p.pool.n_blocks, bad = !there && in_sight(key);
                if (bad) report(p.step, TUTTI_EFAULT);
                missing[i] = __ballot_sync(0xffffffffu, bad);
                tiled = tiled && __all_sync(0xffffffffu, there);
                off[i] = there ? block_offset(p.pool, id[i]) + (int64_t)(p.pool.row_of(key) * p.pool.tok_stride + head * p.pool.head_stride) : -1;
                if constexpr (C8) {
                    const uint64_t at = there ? (uint64_t)id[i] * p.pool.scale_row + head : 0;
                    ks[i] = there ? p.pool.k_scale[at] : 0.0f;
                    vs[i] = there ? p.pool.v_scale[at] : 0.0f;
                }
            }
        };
        if (group == 1) step_unit();
        locate();
        resolve();
        for (uint32_t n = group; fx < x1; n += 2) {     // n: unit of the worker
            // keys behind the end are masked by position, blocks outside the pool by this
            if (lane < 2) exists[(n & 7) * 4 + half * 2 + lane] = ~(lane ? missing[1] : missing[0]);
            uint32_t fac[2][2], sec[2][2];              // 8-bit: the scales' two factors, twice 16 bits
            bool small = false;
            if constexpr (C8) {
                float k_in = 1.0f, v_in = 1.0f;
                if constexpr (C::UNITS) {
                    auto most = [](const float (&x)[2]) {
                        return __reduce_max_sync(0xffffffffu, max(__float_as_uint(fabsf(x[0])), __float_as_uint(fabsf(x[1]))));
                    };
                    const int ku = unit_of(most(ks), UNIT_LEAST_K, UNIT_MOST_K), vu = unit_of(most(vs), UNIT_LEAST_V, UNIT_MOST_V);
                    if (lane == 0) units[(n & 7) * 2 + half] = make_int2(ku, vu);
                    k_in = pow2(-ku);
                    v_in = pow2(-vu);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    small = factors(ks[i] * k_in, fac[0][i], sec[0][i], T()) || small;
                    small = factors(vs[i] * v_in, fac[1][i], sec[1][i], T()) || small;
                }
                small = __any_sync(0xffffffffu, small);
            }
            const bool by_tile = tiled;
            const uint32_t raw_bar = raw_full + 16 * (warp - KV_WARP);
            auto room = [&](int kv) {
                const bool there = n < 2 || mbar_wait(empty + 8 * (2 * group + kv), (n / 2 - 1) & 1, dead);
                return (bool)__all_sync(0xffffffffu, there);
            };
            auto fetch = [&](int kv) {                  // issues the loads of the warp's 64 rows
                const uint32_t dst = base + land[kv];
                if (by_tile) {
                    constexpr uint32_t PARTS = RB / 128 ? RB / 128 : 1;
                    const uint32_t row = my_box * box_rows, bar = C8 ? raw_bar + 8 * kv : full + 8 * (2 * group + kv);
                    const int32_t lo = __shfl_sync(0xffffffffu, id[0], row % 32), hi = __shfl_sync(0xffffffffu, id[1], row % 32);
                    __syncwarp();
                    if (lane == 0) mbar_expect(bar, 64 * RB);
                    __syncwarp();
                    if (my_part < PARTS) {
                        const int32_t token = (int32_t)p.pool.row_of(key_of(key0 + row));
                        tile_load(dst + my_part * ATOM + (half * 64 + row) * 128, kv ? &maps.v : &maps.k, bar, (int32_t)(my_part * (C8 ? 128 : 64)),
                                  p.pool.hnd ? token : (int32_t)head, p.pool.hnd ? (int32_t)head : token, row < 32 ? lo : hi);
                    }
                } else {
                    const uint64_t from = kv ? p.pool.v_base : p.pool.k_base;
#pragma unroll 4
                    for (int it = 0; it < 64 / RPI; ++it) {
                        const uint32_t r = it * RPI + sub, row = half * 64 + r;
                        const int64_t o = __shfl_sync(0xffffffffu, it * RPI < 32 ? off[0] : off[1], r % 32);
                        cp16(dst + (C8 ? row * 128 + (((ch ^ row) & (CH - 1)) << 4) : C::place(row, ch)), (const void *)(from + (o >= 0 ? o : 0) + ch * 16), o >= 0);
                    }
                    cp_commit();
                }
            };
            auto arrive = [&](int kv) {                 // the warp's rows are in their places
                fence_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(full + 8 * (2 * group + kv));
            };
            // 8-bit: four steps' codes are read before the rows they may lie in are written
            auto widen = [&](int kv, uint32_t fa, uint32_t fb, uint32_t sa, uint32_t sb, auto two_factors) {
                constexpr int B = 4;
                const unsigned char *src = sm + (kv ? land[1] : land[0]);
                unsigned char *dst = sm + slot0 + kv * C::KV;
#pragma unroll 1
                for (int it0 = 0; it0 < 64 / RPI; it0 += B) {
                    uint4 c[B];
                    uint32_t top = 0;
#pragma unroll
                    for (int k = 0; k < B; ++k) {
                        const uint32_t row = half * 64 + (it0 + k) * RPI + sub;
                        c[k] = *reinterpret_cast<const uint4 *>(src + row * 128 + (((ch ^ row) & (CH - 1)) << 4));
                    }
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < B; ++k) {
                        const uint32_t r = (it0 + k) * RPI + sub, row = half * 64 + r;
                        const uint32_t f1 = __shfl_sync(0xffffffffu, r < 32 ? fa : fb, r % 32);
                        const uint32_t w[4] = {c[k].x, c[k].y, c[k].z, c[k].w};
                        uint32_t e[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint2 x = spread(w[i], T(), top);
                            e[2 * i] = times(x.x, f1, T());
                            e[2 * i + 1] = times(x.y, f1, T());
                        }
                        if constexpr (two_factors.value) {
                            const uint32_t f2 = __shfl_sync(0xffffffffu, r < 32 ? sa : sb, r % 32);
#pragma unroll
                            for (int i = 0; i < 8; ++i) e[i] = times(e[i], f2, T());
                        }
                        *reinterpret_cast<uint4 *>(dst + C::place(row, 2 * ch)) = make_uint4(e[0], e[1], e[2], e[3]);
                        *reinterpret_cast<uint4 *>(dst + C::place(row, 2 * ch + 1)) = make_uint4(e[4], e[5], e[6], e[7]);
                    }
                    if (C::ORDERED ? false : __vmaxu2(top, 0x07e007e0u) != 0x07e007e0u) {       // NaN codes: they are made NaN again
#pragma unroll
                        for (int k = 0; k < B; ++k) {
                            const uint32_t row = half * 64 + (it0 + k) * RPI + sub;
                            const uint32_t w[4] = {c[k].x, c[k].y, c[k].z, c[k].w};
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                // code i of the 16 is element {0, 2, 1, 3}[i % 4] of its four
                                const int e = (i & ~3) | (i & 1) << 1 | (i >> 1 & 1);
                                if ((w[i / 4] >> (8 * (i & 3)) & 0x7f) == 0x7f)
                                    *reinterpret_cast<uint16_t *>(dst + C::place(row, 2 * ch + e / 8) + (e % 8) * 2) = 0x7fff;
                            }
                        }
                    }
                }
            };
            if constexpr (!C8) {
#pragma unroll 1
                for (int kv = 0; kv < 2 && (ok = room(kv)); ++kv) fetch(kv);
                if (!ok) break;
#pragma unroll 1
                for (int k = 0; k < 2; ++k) step_unit();
                locate();                               // the next unit's ids arrive while this one's rows do
                if (!by_tile) {                         // tensor copies arrive at `full` by themselves
                    cp_wait<1>();
                    arrive(0);
                    cp_wait<0>();
                    arrive(1);
                }
                resolve();
            } else {
                fetch(1);
                if (!(ok = room(0))) break;
                fetch(0);
                step_unit();
                step_unit();
                locate();
#pragma unroll 1                                        // the widening loops once in the code: 265 us against 293 on the 8-bit chunk of the header (fetching of instructions)
                for (int kv = 0; kv < 2; ++kv) {
                    if (kv == 1) {
                        resolve();                      // the next unit's scales arrive while this one's values are widened
                        if (!(ok = room(1))) break;
                    }
                    if (by_tile) {
                        ok = mbar_wait(raw_bar + 8 * kv, raw_phase & 1, dead);
                        if (!(ok = __all_sync(0xffffffffu, ok))) break;
                    } else {
                        cp_wait<0>();
                        __syncwarp();                   // the warp's rows, brought by all its lanes
                    }
                    const uint32_t fa = kv ? fac[1][0] : fac[0][0], fb = kv ? fac[1][1] : fac[0][1];
                    const uint32_t sa = kv ? sec[1][0] : sec[0][0], sb = kv ? sec[1][1] : sec[0][1];
                    if (small) widen(kv, fa, fb, sa, sb, std::true_type());
                    else widen(kv, fa, fb, sa, sb, std::false_type());
                    arrive(kv);
                }
                if (!ok) break;
                if (by_tile) ++raw_phase;
            }
        }
        cp_wait<0>();
        } else if (warp >= Q_WARP) {
        // =================================== queries ===================================
        uint32_t segs = 0;
        for (unsigned long long x = x0; x < x1; ++segs) {
            const uint32_t n = (uint32_t)min(x1 - x, (unsigned long long)(t.n_units - t.u));
            bool ok = warp != Q_WARP || segs < SHARES || mbar_wait(share_free + 8 * (segs % SHARES), (segs / SHARES - 1) & 1, dead);
            if (!__all_sync(0xffffffffu, ok)) break;
            if (warp == Q_WARP && lane == 0) {
                shares[segs % SHARES] = Share{n, t.u, t.n_units, shift_of(t), t.q, t.h, t.v.q0, t.r.n_rows, t.r.first};
                mbar_arrive(share_full + 8 * (segs % SHARES));
            }
            ok = !segs || mbar_wait(q_empty, (segs - 1) & 1, dead);
            if (!__all_sync(0xffffffffu, ok)) break;
            constexpr int CH = D / 8, RPI = 32 / CH;        // 16-byte chunks of a row; rows a warp takes at once
            const uint32_t ch = lane % CH, sub = lane / CH;
#pragma unroll 1
            for (uint32_t b = warp - Q_WARP; b < TILE_ROWS / 32; b += Q_WARPS) {
                const uint32_t mine = t.q * TILE_ROWS + b * 32 + lane;
                const bool in = mine < t.r.n_rows;          // zeros behind the last row
                const uint32_t k = in ? p.token_of(mine) : 0, h = t.h * p.group + (in ? p.member_of(mine) : 0);
                const uint64_t src = in ? (uint64_t)((const T *)p.q + (uint64_t)(t.v.q0 + k) * p.q_stride + (uint64_t)h * D) : 0;
#pragma unroll
                for (uint32_t it = 0; it < CH; ++it) {
                    const uint32_t r = b * 32 + it * RPI + sub;
                    const uint64_t from = __shfl_sync(0xffffffffu, src, r % 32);
                    cp16(base + r / HALF_ROWS * C::KV + C::place(r % HALF_ROWS, ch), (const void *)((from ? from : (uint64_t)p.q) + ch * 16), from != 0);
                }
            }
            cp_commit();
            cp_wait<0>();
            if (!C::ORDERED || p.scale < 0) {               // each lane what it brought itself
                const uint32_t sign = p.scale < 0 ? 0x80008000u : 0;
#pragma unroll 1
                for (uint32_t b = warp - Q_WARP; b < TILE_ROWS / 32; b += Q_WARPS)
#pragma unroll 4
                    for (uint32_t it = 0; it < CH; ++it) {
                        const uint32_t r = b * 32 + it * RPI + sub;
                        uint4 *at = reinterpret_cast<uint4 *>(sm + r / HALF_ROWS * C::KV + C::place(r % HALF_ROWS, ch));
                        uint4 u = *at;
                        if constexpr (!C::ORDERED)
                            u = make_uint4(__byte_perm(u.x, u.y, 0x5410), __byte_perm(u.x, u.y, 0x7632), __byte_perm(u.z, u.w, 0x5410), __byte_perm(u.z, u.w, 0x7632));
                        *at = make_uint4(u.x ^ sign, u.y ^ sign, u.z ^ sign, u.w ^ sign);
                    }
            }
            fence_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
            x += n;
            if (x < x1) next_tile(p, t);
        }
        cp_wait<0>();
        } else {
        // =================================== matrix instructions ===================================
        {
            // the warp stays together; one elected lane issues, so operands live in uniform registers
            constexpr uint32_t FMT = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
            constexpr uint32_t IDESC = 1u << 4 | FMT << 7 | FMT << 10 | (uint32_t)(HALF_ROWS / 16) << 24;
            constexpr uint32_t ID_QK = IDESC | (uint32_t)(SUB / 8) << 17, ID_PV = IDESC | 1u << 16 | (uint32_t)(D / 8) << 17;
            uint32_t n_unit = 0, segs = 0, np[2] = {0, 0}, ns[2] = {0, 0};
            bool ok = true;
            constexpr uint32_t STEP_BYTES = SUB * 128;          // from a step's rows to the next one's
            auto qk = [&](int i, int u, uint32_t slot) {
                const uint64_t a = operand(base + i * C::KV), b = operand(base + C::OFF_RING + slot * C::KV + u * STEP_BYTES);
                if (elect()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t step = ((k / 4) * ATOM + (k % 4) * 32) >> 4;
                        mma_ss(S(i, u), a + step, b + step, ID_QK, k > 0);
                    }
                    tc_commit(s_full + 8 * (2 * i + u));
                }
                __syncwarp();
            };
            auto pv = [&](int i, int u, uint32_t slot, bool acc) {
                const uint64_t b = operand(base + C::OFF_RING + slot * C::KV + u * STEP_BYTES);
                if (elect()) {
#pragma unroll
                    for (int k = 0; k < SUB / 16; ++k) mma_ts(O(i), S(i, u) + k * 8, b + ((k * 2048) >> 4), ID_PV, acc || k > 0);
                    tc_commit(o_full + 8 * i);
                }
                __syncwarp();
            };
            auto commit = [&](uint32_t bar) {
                if (elect()) tc_commit(bar);
                __syncwarp();
            };
            // K (0) or V (1) of unit u of the worker
            auto slot = [](uint32_t u, uint32_t kv) { return (u & 1) * 2 + kv; };
            auto all = [](bool x) { return (bool)__all_sync(0xffffffffu, x); };
            auto landed = [&](uint32_t u, uint32_t kv) { return mbar_wait(full + 8 * slot(u, kv), (u / 2) & 1, dead); };
            for (unsigned long long x = x0; x < x1 && ok;) {
                ok = all(mbar_wait(q_full, segs & 1, dead) && landed(n_unit, 0));
                if (!ok) break;
                const Share &t = shares[segs % SHARES];         // published before the queries were brought
                const uint32_t n = t.n;
                const int halves = t.n_rows - t.q * TILE_ROWS > HALF_ROWS ? 2 : 1;
                tc_after();
                for (int u = 0; u < STEPS; ++u)
                    for (int i = 0; i < halves; ++i) qk(i, u, slot(n_unit, 0));
                commit(empty + 8 * slot(n_unit, 0));
                if (n == 1) commit(q_empty);            // behind the last Q K^T of the tile
                x += n;
                for (uint32_t j = 0; j < n && ok; ++j, ++n_unit) {
                    const bool more = j + 1 < n;
                    ok = all(landed(n_unit, 1) && (!more || landed(n_unit + 1, 0)));
                    for (int u = 0; u < STEPS && ok; ++u)
                        for (int i = 0; i < halves && ok; ++i) {
                            ok = mbar_wait(p_full + 8 * (2 * i + u), np[i] & 1, dead);
                            if (ok && j == 0 && u == 0 && ns[i]) ok = mbar_wait(o_empty + 8 * i, (ns[i] - 1) & 1, dead);
                            if (!(ok = all(ok))) break;
                            tc_after();
                            pv(i, u, slot(n_unit, 1), j > 0 || u > 0);
                            if (more) qk(i, u, slot(n_unit + 1, 0));
                            else if (u == STEPS - 1) commit(o_done + 8 * i);
                            np[i] += u == STEPS - 1;
                        }
                    if (!ok) break;
                    commit(empty + 8 * slot(n_unit, 1));
                    if (more) commit(empty + 8 * slot(n_unit + 1, 0));
                    if (j + 2 == n) commit(q_empty);
                }
                if (!ok) break;
                for (int i = 0; i < halves; ++i) ++ns[i];
                ++segs;
            }
            // every matrix instruction has ended before TMEM is given back
            commit(drain);
            const long long t0 = clock64();
            while (!mbar_try(drain, 0) && clock64() - t0 < WAIT_CLOCKS) {}
        }
        __syncwarp();
        }
    } else {
        // =================================== softmax ===================================
        setmaxnreg_inc<C::SOFT_REGS>();
        const int i = warp / 4;                                   // half
        const uint32_t lanes = (warp % 4) * 32 << 16, o_at = O(i) + lanes, r = (warp % 4) * 32 + lane;
        // Scores are multiplied by a positive factor (a negative scale's sign is on the queries), so that masked ones stay
        // -infinity and the largest stays the largest; the smallest number there is makes the largest score of a zero scale less than 2^-20.
        const float scl_all = fmaxf(fabsf(p.scale) * 1.4426950408889634f, 0x1p-149f);
        uint32_t n_s = 0, n_seg = 0, n_unit = 0, n_join = 0, n_share = 0;    // steps of this half; units of the worker
        bool ok = true;
        auto join = [&]() {                                       // the half's four warps
            __syncwarp();
            if (lane == 0) mbar_arrive(joined + 8 * i);
            const bool there = mbar_wait(joined + 8 * i, n_join++ & 1, dead);
            return (bool)__all_sync(0xffffffffu, there);
        };
        for (unsigned long long x = x0; x < x1 && ok;) {
            ok = mbar_wait(share_full + 8 * (n_share % SHARES), n_share / SHARES & 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const Share t = shares[n_share % SHARES];
            __syncwarp();
            if (lane == 0) mbar_arrive(share_free + 8 * (n_share % SHARES));
            ++n_share;
            const uint32_t n = t.n;
            const uint32_t row = t.q * TILE_ROWS + i * HALF_ROWS + r;
            if (t.q * TILE_ROWS + i * HALF_ROWS < t.n_rows) {
                const bool in = row < t.n_rows;
                // rows behind the last take the last one's position: they are computed and dropped
                const uint32_t tok = p.token_of(in ? row : t.n_rows - 1);
                const int64_t pos = t.first + tok;
                const int64_t pos_low = __shfl_sync(0xffffffffu, pos, 0);
                const int64_t hidden = WIN ? __shfl_sync(0xffffffffu, pos, 31) - p.window : 0;      // keys up to here are not seen by every row
                float m = -INFINITY, l = 0;
                int o_unit = UNIT_LEAST_V;                        // UNITS: exponent of the output's unit, the largest of its values'
                const uint32_t steps = STEPS * n;
                for (uint32_t j = 0; j < steps && ok; ++j) {
                    const int u = j % STEPS;
                    const uint32_t s_at = S(i, u) + lanes;
                    ok = mbar_wait(s_full + 8 * (2 * i + u), n_s / STEPS & 1, dead);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_after();
                    uint32_t sr[SUB];
                    float *s = reinterpret_cast<float *>(sr);
#pragma unroll
                    for (int q = 0; q < SUB / 32; ++q) tc_ld32(sr + 32 * q, s_at + 32 * q);
                    uint32_t ex[SUB / 32], all = ~0u;             // keys that exist
#pragma unroll
                    for (int q = 0; q < SUB / 32; ++q) {
                        ex[q] = exists[((n_unit + j / STEPS) & 7) * 4 + SUB / 32 * u + q];
                        all &= ex[q];
                    }
                    float scl = scl_all;
                    int below = 0;                                // of the values' unit to the output's
                    if constexpr (C::UNITS) {
                        const int2 unit = units[((n_unit + j / STEPS) & 7) * 2 + u];
                        scl = fmaxf(scl * pow2(unit.x), 0x1p-126f);         // not zero, for the scores of -infinity
                        below = o_unit - unit.y;
                    }
                    tc_wait_ld();
#pragma unroll
                    for (int q = 0; q < SUB / 32; ++q) tc_loaded(sr + 32 * q);
                    const int64_t v0 = (int64_t)t.u * BN + j * SUB, key0 = WIN ? v0 + t.shift : v0;    // (of numbers below p.front: v0)
                    if (key0 + SUB - 1 > pos_low || all != ~0u || (WIN && key0 <= hidden)) {
                        // A bit a key, and two instructions a score: this code runs once or twice a tile, so that it is fetched
                        // each time (with three comparisons a score a masked unit took 9 us instead of 2).
                        auto ahead = [](int64_t n) { return n < 0 ? 0 : n > SUB ? SUB : (int)n; };
                        auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; };       // bits 0 .. n - 1
                        const int seen = ahead(pos - key0 + 1), gone = WIN ? ahead(pos - p.window - key0 + 1) : 0;
                        // WIN: the sequence's first tokens, which all rows see; where a shift begins behind `front`, they are in front of it
                        const int cut = WIN && t.shift ? ahead((int64_t)p.front - v0) : 0;
                        const int first = WIN ? min(ahead((int64_t)p.sinks - v0), t.shift ? cut : seen) : 0;
#pragma unroll
                        for (int q = 0; q < SUB / 32; ++q) {
                            uint32_t bits = below(seen - 32 * q);
                            if constexpr (WIN) bits = (bits & ~below(gone - 32 * q) & ~below(cut - 32 * q)) | below(first - 32 * q);
                            bits &= ex[q];
#pragma unroll
                            for (int k = 0; k < 32; ++k) s[32 * q + k] = bits & 1u << k ? s[32 * q + k] : -INFINITY;
                        }
                    }
                    float a0 = max3(s[0], s[4], s[8]), a1 = max3(s[1], s[5], s[9]), a2 = max3(s[2], s[6], s[10]), a3 = max3(s[3], s[7], s[11]);
#pragma unroll
                    for (int k = 12; k < SUB - 4; k += 8) {
                        a0 = max3(a0, s[k], s[k + 4]);
                        a1 = max3(a1, s[k + 1], s[k + 5]);
                        a2 = max3(a2, s[k + 2], s[k + 6]);
                        a3 = max3(a3, s[k + 3], s[k + 7]);
                    }
                    a0 = max3(a0, s[SUB - 4], s[SUB - 3]);
                    a1 = max3(a1, s[SUB - 2], s[SUB - 1]);
                    const float top = max3(a0, a1, fmaxf(a2, a3)) * scl;
                    const bool grow = top > m + GROW || (m == -INFINITY && top > m);
                    if (__any_sync(0xffffffffu, grow) || below != 0) {          // rare: the reference has to move, or the unit
                        float alpha = grow ? ex2(m - top) : 1.0f;
                        if (grow) m = top;
                        l *= alpha;
                        if (below != 0) {                         // exact, and far from the ends of the range
                            alpha *= pow2(below);
                            o_unit -= below;
                        }
                        if (j > 0) {
                            // these scores were issued behind the product two steps back, so only the last one's may be open
                            ok = mbar_wait(o_full + 8 * i, (n_s - 1) & 1, dead);
                            ok = __all_sync(0xffffffffu, ok);
                            if (!ok) break;
                            tc_after();
#pragma unroll 1
                            for (int q = 0; q < D / 16; ++q) {
                                uint32_t o[16];
                                tc_ld16(o, o_at + 16 * q);
                                tc_wait_ld();
                                asm volatile("" : P4(o, 0), P4(o, 4), P4(o, 8), P4(o, 12));
#pragma unroll
                                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                                tc_st16(o, o_at + 16 * q);
                            }
                        }
                    }
                    // Exponentials against the reference; their 32-bit sums go to l, and 16 bits of each over the scores:
                    // the matrix instruction takes P and V of one 16-bit type.  (bf16: the outputs of the chunk above
                    // are off from 64-bit arithmetic by 0.0023 of their size instead of 0.0017, what rounding them costs.)
                    const float sub = C::OFF - (m == -INFINITY ? 0.0f : m);
                    const f2 scl2 = pair(scl, scl), sub2 = pair(sub, sub);
                    f2 l0 = 0, l1 = 0;
#pragma unroll
                    for (int q = 0; q < SUB / 32; ++q) {
                        uint32_t pk[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float a, b;
                            unpair(fma2(pair(s[32 * q + 2 * k], s[32 * q + 2 * k + 1]), scl2, sub2), a, b);
                            a = ex2(a);
                            b = ex2(b);
                            if (k & 1) l1 = add2(l1, pair(a, b));
                            else l0 = add2(l0, pair(a, b));
                            pk[k] = pack2(a, b, T());
                        }
                        tc_st16(pk, s_at + 16 * q);
                    }
                    float la, lb;
                    unpair(add2(l0, l1), la, lb);
                    l += la + lb;
                    tc_wait_st();
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 8 * (2 * i + u));
                    ++n_s;
                }
                if (!ok) break;
                // (o_full would not do: two of its phases may be open here, and one bit does not tell them apart)
                ok = mbar_wait(o_done + 8 * i, n_seg++ & 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_after();
                if (C::UNITS && o_unit != UNIT_LEAST_V) {          // outputs 2^x too small: as much in the reference, out of the sum
                    m += (float)(o_unit - UNIT_LEAST_V);
                    l *= pow2(UNIT_LEAST_V - o_unit);
                }
                const bool whole = t.u == 0 && n == t.n_units;
                uint32_t w0 = 0, w1 = 0;
                if (!whole) holders(x - t.u, t.n_units, workers, total, w0, w1);
            // Outputs in pieces of 32 dimensions, by loops that are not unrolled: a tile's end is code that has to be fetched, and
            // all 128 at once spilled 1 KB a thread (8 us from a tile's last score to the next one's first; so 5).
            auto outputs = [&](uint32_t q, float (&o)[32]) {
                tc_ld32(reinterpret_cast<uint32_t *>(o), o_at + 32 * q);
                tc_wait_ld();
                tc_loaded(reinterpret_cast<uint32_t *>(o));
            };
            auto given_back = [&]() {                              // the outputs' place
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_empty + 8 * i);
            };
            bool write = true;
            auto slot = [&](uint32_t k) { return (k == w0 ? 2 * k + 1 : 2 * k) * 2 + i; };
            float4 *part = reinterpret_cast<float4 *>(ws.part);
            float2 *ml = reinterpret_cast<float2 *>(ws.part + (uint64_t)4 * ws.workers * HALF_ROWS * D);
            auto at = [&](uint32_t k, uint32_t d4) { return part + ((uint64_t)slot(k) * (D / 4) + d4) * HALF_ROWS + r; };
            if (!whole) {
#pragma unroll 1
                for (uint32_t q = 0; q < D / 32; ++q) {
                    float o[32];
                    outputs(q, o);
#pragma unroll
                    for (uint32_t d = 0; d < 8; ++d) *at(w, 8 * q + d) = make_float4(o[4 * d], o[4 * d + 1], o[4 * d + 2], o[4 * d + 3]);
                }
                ml[(uint64_t)slot(w) * HALF_ROWS + r] = make_float2(m, l);
                given_back();
                if (!(ok = join())) break;
                if (r == 0) {
                    const uint32_t old = arrive_gpu(ws.count + 2 * w0 + i);
                    if (old == w1 - w0) ws.count[2 * w0 + i] = 0;            // ready for the next call
                    misc[74 + i] = old == w1 - w0;
                }
                if (!(ok = join())) break;
                write = *(volatile uint32_t *)(misc + 74 + i);
                if (write) {
                m = -INFINITY;
                l = 0;
#pragma unroll 4
                for (uint32_t k = w0; k <= w1; ++k) m = fmaxf(m, __ldcg(ml + (uint64_t)slot(k) * HALF_ROWS + r).x);
#pragma unroll 4
                for (uint32_t k = w0; k <= w1; ++k) {
                    const float2 e = __ldcg(ml + (uint64_t)slot(k) * HALF_ROWS + r);
                    l += e.y * (m == -INFINITY ? 0.0f : ex2(e.x - m));
                }
                }
            }
            if (write) {
            const uint64_t token = t.q0 + tok;
            const uint32_t qh = t.h * p.group + p.member_of(in ? row : t.n_rows - 1);
            const unsigned long long out_row = in ? (unsigned long long)((T *)p.out + token * p.out_stride + (uint64_t)qh * D) : 0;
            float *lse_at = p.lse && in ? p.lse + token * p.n_q_heads + qh : nullptr;
            // l, not m, tells a row that saw nothing: scores of NaN move no maximum, but make the sum NaN
            const float inv = l == 0 ? 0.0f : (C::UNITS ? pow2(UNIT_LEAST_V) : 1.0f) / l;
            unsigned long long to[4];                              // the rows of the lane's quad
#pragma unroll
            for (int k = 0; k < 4; ++k) to[k] = __shfl_sync(0xffffffffu, out_row, (lane & ~3u) + k);
#pragma unroll 1
            for (uint32_t q = 0; q < D / 32; ++q) {
                float o[32];
                if (whole) {
                    outputs(q, o);
                } else {                                           // the parts in worker order
#pragma unroll
                    for (int d = 0; d < 32; ++d) o[d] = 0;
#pragma unroll 2
                    for (uint32_t k = w0; k <= w1; ++k) {
                        float4 b[8];
                        const float2 e = __ldcg(ml + (uint64_t)slot(k) * HALF_ROWS + r);
#pragma unroll
                        for (uint32_t d = 0; d < 8; ++d) b[d] = __ldcg(at(k, 8 * q + d));
                        const float c = m == -INFINITY ? 0.0f : ex2(e.x - m);
#pragma unroll
                        for (uint32_t d = 0; d < 8; ++d)
                            o[4 * d] += b[d].x * c, o[4 * d + 1] += b[d].y * c, o[4 * d + 2] += b[d].z * c, o[4 * d + 3] += b[d].w * c;
                    }
                }
                // A thread has a row, a store wants neighbouring lanes on neighbouring bytes: the four lanes
                // of a quad exchange 16-byte pieces, so that a store writes 64 bytes of a row (a piece of its
                // own row a lane made a store of 32 separate lines: 3 us a tile, and the load of the next
                // tile's queries behind it)
                uint32_t piece[4][4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    constexpr int B = C::ORDERED ? 1 : 2, E = C::ORDERED ? 2 : 1;      // where elements 1 and 2 of four are
                    const float *e = o + 8 * k;
                    piece[k][0] = pack2(e[0] * inv, e[B] * inv, T()), piece[k][1] = pack2(e[E] * inv, e[3] * inv, T());
                    piece[k][2] = pack2(e[4] * inv, e[4 + B] * inv, T()), piece[k][3] = pack2(e[4 + E] * inv, e[7] * inv, T());
                }
                // (row, piece) to (piece, row): the off-diagonal blocks change places, at distance 2 and 1
#pragma unroll
                for (int dist = 2; dist; dist >>= 1)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k & dist) continue;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool up = lane & dist;
                            const uint32_t give = up ? piece[k][e] : piece[k + dist][e];
                            const uint32_t got = __shfl_xor_sync(0xffffffffu, give, dist);
                            if (up) piece[k][e] = got;
                            else piece[k + dist][e] = got;
                        }
                    }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (to[k]) *reinterpret_cast<uint4 *>(to[k] + (4 * q + (lane & 3)) * 16) = make_uint4(piece[k][0], piece[k][1], piece[k][2], piece[k][3]);
            }
            if (lse_at) *lse_at = l == 0 ? -INFINITY : (m - C::OFF + log2f(l)) * 0.6931471805599453f;
            if (whole) given_back();
            }
            }
            n_unit += n;
            x += n;
        }
    }
    if (*dead) {                                    // a wait was given up: copies in flight get 1 ms to land
        const long long t0 = clock64();
        while (clock64() - t0 < WAIT_CLOCKS / 1500) {}
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (threadIdx.x == 0 && *dead) report(p.step, TUTTI_ETIMEDOUT);
    if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <typename T, bool C8, int D>
cudaError_t launch(const AttendParams &p, const PoolMaps &maps, const Workspace &ws, cudaStream_t st) {
    return p.window ? launch_behind(attend_many_kernel<T, C8, D, true>, ws.workers, THREADS, Many<T, C8, D>::SMEM, st, p, maps, ws)
                    : launch_plain(attend_many_kernel<T, C8, D, false>, ws.workers, THREADS, Many<T, C8, D>::SMEM, st, p, maps, ws);
}

template <typename T, bool C8>
cudaError_t launch(const AttendParams &p, const PoolMaps &maps, const Workspace &ws, cudaStream_t st) {
    return p.pool.head_dim == 128 ? launch<T, C8, 128>(p, maps, ws, st) : launch<T, C8, 64>(p, maps, ws, st);
}

template <typename T, bool C8, int D>
cudaError_t setup() {
    const cudaError_t e = cudaFuncSetAttribute(attend_many_kernel<T, C8, D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Many<T, C8, D>::SMEM);
    return e == cudaSuccess ? cudaFuncSetAttribute(attend_many_kernel<T, C8, D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Many<T, C8, D>::SMEM) : e;
}

template <typename T>
cudaError_t setup_type() {
    cudaError_t e = setup<T, false, 128>();
    if (e == cudaSuccess) e = setup<T, true, 128>();
    if (e == cudaSuccess) e = setup<T, false, 64>();
    if (e == cudaSuccess) e = setup<T, true, 64>();
    return e;
}

}  // namespace

cudaError_t many_setup() {
    const cudaError_t e = setup_type<__nv_bfloat16>();
    return e == cudaSuccess ? setup_type<__half>() : e;
}

cudaError_t many_launch(const AttendParams &p, const PoolMaps &maps, const Workspace &ws, bool c8, bool bf, cudaStream_t st) {
    if (c8) return bf ? launch<__nv_bfloat16, true>(p, maps, ws, st) : launch<__half, true>(p, maps, ws, st);
    return bf ? launch<__nv_bfloat16, false>(p, maps, ws, st) : launch<__half, false>(p, maps, ws, st);
}

uint32_t many_workers(int sms) { return (uint32_t)sms; }
size_t many_part_bytes(uint32_t workers) { return (size_t)4 * workers * HALF_ROWS * (128 + 2) * sizeof(float); }

}  // namespace tutti

// The kernel's functions for cuts and parts, on the host, over tiles of n_units[i] units laid end to end (the search
// for the tile of a cut is the caller's): the share [x0, x1) of worker w; and for a tile the first and the last worker
// that has a part of it.
extern "C" void tutti_many_cut_(const uint32_t *n_units, uint32_t n_tiles, uint64_t workers, uint64_t w, uint64_t *out) {
    uint64_t total = 0;
    for (uint32_t i = 0; i < n_tiles; ++i) total += n_units[i];
    for (int c = 0; c < 2; ++c) {
        const uint64_t x = tutti::cut_of(w + c, workers, total);
        uint64_t at = 0;
        uint32_t i = 0;
        while (i < n_tiles && x >= at + n_units[i]) at += n_units[i++];
        out[c] = i < n_tiles ? at + tutti::snapped((uint32_t)(x - at), n_units[i]) : x;
    }
}
extern "C" void tutti_many_parts_(uint64_t tile0, uint32_t n, uint64_t workers, uint64_t total, uint64_t *out) {
    uint32_t w0, w1;
    tutti::holders(tile0, n, workers, total, w0, w1);
    out[0] = w0;
    out[1] = w1;
}

// The kernel's own count of units, on the host: out2[0] units of tile q, out2[1] units of the tiles before it.
static void tile_params(tutti::AttendParams &p, uint32_t group, uint32_t window, uint32_t sinks, uint32_t block_tokens) {
    p.group = group;
    tutti::division_by(group, p.group_mul, p.group_shift);
    p.window = window;
    p.sinks = sinks;
    p.grain = tutti::grain_of(block_tokens);
    p.front = tutti::front_of(sinks, p.grain);
}
extern "C" int tutti_many_units_(uint32_t ctx, uint32_t n_new, uint32_t group, uint32_t q, uint64_t *out2) {
    const tutti::SeqView v{0, n_new, ctx, 0};
    tutti::AttendParams p;
    tile_params(p, group, 0, 0, 16);
    tutti::Rows r;
    tutti::rows_of(v, p, r);
    out2[0] = q < r.n_tiles ? r.units(q) : 0;
    out2[1] = r.before(q);
    return (int)r.n_tiles;
}
// The same under a window; out4[2] the sequence's first keys that a tile has, out4[3] its shift of the others.
extern "C" int tutti_many_window_units_(uint32_t ctx, uint32_t n_new, uint32_t group, uint32_t window, uint32_t sinks, uint32_t block_tokens, uint32_t q, uint64_t *out4) {
    const tutti::SeqView v{0, n_new, ctx, 0};
    tutti::AttendParams p;
    tile_params(p, group, window, sinks, block_tokens);
    tutti::WindowRows r;
    tutti::rows_of(v, p, r);
    out4[0] = q < r.n_tiles ? r.units(q) : 0;
    out4[1] = r.before(q);
    out4[2] = r.front;
    out4[3] = q < r.n_tiles ? r.shift(q) : 0;
    return (int)r.n_tiles;
}

// What a code becomes on its way into a many-row product, on the host: the two 16-bit elements of a pair (one
// code twice) behind both factors, as `widen` multiplies them.  f16: in the unit that a step whose largest
// scale is `top` has (its exponent goes to *unit; keys or values by their least one).
template <typename T>
static uint32_t widened(uint8_t code, float scale) {
    __nv_fp8_e4m3 c;
    c.__x = code;
    const float start = std::is_same<T, __half>::value ? (float)c : (float)c * 0x1p-120f;      // see spread()
    uint32_t f1, f2;
    const bool two = tutti::factors(scale, f1, f2, T());
    const uint32_t x = tutti::times(tutti::twice(start, T()), f1, T());
    return two ? tutti::times(x, f2, T()) : x;
}
extern "C" uint32_t tutti_many_widen_(uint32_t code, float scale, float top, uint32_t dtype, uint32_t is_v, int32_t *unit) {
    *unit = 0;
    if (dtype == TUTTI_DTYPE_BF16) return widened<__nv_bfloat16>((uint8_t)code, scale);
    uint32_t bits;
    memcpy(&bits, &top, 4);
    *unit = is_v ? tutti::unit_of(bits, tutti::UNIT_LEAST_V, tutti::UNIT_MOST_V) : tutti::unit_of(bits, tutti::UNIT_LEAST_K, tutti::UNIT_MOST_K);
    return widened<__half>((uint8_t)code, scale * tutti::pow2(-*unit));
}
