// Attention of many rows per sequence (a prompt chunk behind a restored prefix, a speculative
// step): both products on the 5th-generation tensor cores.
//
// A *tile* is 256 rows of one sequence and KV head, two halves of 128 rows (the M of one
// tcgen05.mma), against keys in units of 128.  As in the few-row kernel all units of all tiles
// are dealt out evenly over the SMs, one worker (CTA) each, and a tile that several workers share
// is joined by the last of them; a causal tile's units are counted in closed form (floor_sum), so
// a captured graph follows lengths that change.
//
// Roles of a worker's 12 warps:
//   0-3, 4-7  softmax of half 0 / half 1: a thread owns a row, reads its scores from TMEM, writes
//             its probabilities back over them (16 bits), rescales the output when the running
//             maximum has grown by more than 2^8, and writes the row out at the end;
//   8         issues the matrix instructions: S = Q K^T (both operands in shared memory),
//             O += P V (P from TMEM).  The halves alternate, so the tensor cores work on one
//             while the other is in its softmax;
//   9-11      gather keys and values through the block table into a ring of four 128-row tiles
//             in the 128-byte swizzle (K: K-major B operand, V: the same bytes read as an
//             MN-major B operand).  8-bit codes become 16-bit elements on the way: code * scale,
//             exact for the powers of two that append writes.
// Bound: the tensor cores (2 x 128 x 128 x D multiply-adds a half and unit) and, as close,
// the 128 x 128 exponentials on 16 lanes a clock.
#include <type_traits>

#include "tutti_attend.h"

namespace tutti {

namespace {

constexpr int HALF_ROWS = 128;
constexpr int TILE_ROWS = 256;
constexpr int BN = 128;                 // keys of a unit
constexpr int RING = 4;                 // K and V tiles in flight
constexpr int THREADS = 384;
constexpr int MMA_WARP = 8, PROD_WARP = 9, PROD_WARPS = 3;
constexpr uint32_t ATOM = BN * 128;     // 128 rows of 128 bytes
constexpr float GROW = 8.0f;            // log2 of how far probabilities may exceed 1
constexpr long long WAIT_CLOCKS = 3000000000ll;   // about 1.5 s: a wait that takes longer is given up

// sum over i in [0, n) of floor((a i + b) / m)  (a, b >= 0, m > 0)
__host__ __device__ inline uint64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b) {
    uint64_t ans = 0;
    while (n) {
        if (a >= m) {
            ans += n * (n - 1) / 2 * (a / m);
            a %= m;
        }
        if (b >= m) {
            ans += n * (b / m);
            b %= m;
        }
        const uint64_t y = a * n + b;
        if (y < m) break;
        n = y / m;
        b = y % m;
        const uint64_t t = m;
        m = a;
        a = t;
    }
    return ans;
}

// The tiles of one sequence and head.
struct Rows {
    uint32_t n_rows, n_tiles, group, ctx;
    int64_t first;                      // position of the first new token
    // units of tile q: up to the key of its last row
    __host__ __device__ uint32_t units(uint32_t q) const {
        if (first < 0 || ctx == 0) return ctx ? (ctx + BN - 1) / BN : 1;     // padding rows: every tile sees all
        const uint64_t end = (uint64_t)(q + 1) * TILE_ROWS < n_rows ? (uint64_t)(q + 1) * TILE_ROWS : n_rows;
        return (uint32_t)(((uint64_t)first + (end - 1) / group) / BN) + 1;
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

__host__ __device__ inline Rows rows_of(const SeqView &v, uint32_t group) {
    Rows r;
    r.n_rows = v.n_new * group;
    r.n_tiles = (r.n_rows + TILE_ROWS - 1) / TILE_ROWS;
    r.group = group;
    r.ctx = v.ctx;
    r.first = (int64_t)v.ctx - v.n_new;
    return r;
}

struct Tile {
    uint32_t s, h, q, u, n_units;
    SeqView v;
    Rows r;
};

__device__ inline int tile_seq(const AttendParams &p, uint32_t s, Tile &t) {
    t.s = s;
    const int code = seq_view(p.step, p.pool.block_tokens, s, t.v);
    if (code != TUTTI_OK) t.v.n_new = t.v.ctx = 0;
    t.r = rows_of(t.v, p.group);
    return code;
}

__device__ inline void next_tile(const AttendParams &p, Tile &t) {
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
__device__ inline void tc_st32(const uint32_t *r, uint32_t a) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 ::I4(r, 0), I4(r, 4), I4(r, 8), I4(r, 12), I4(r, 16), I4(r, 20), I4(r, 24), I4(r, 28), "r"(a) : "memory");
}
__device__ inline void tc_st16(const uint32_t *r, uint32_t a) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::I4(r, 0), I4(r, 4), I4(r, 8), I4(r, 12), "r"(a) : "memory");
}

// Shared-memory operand in the 128-byte swizzle: start, offset between 64-element groups of an
// MN-major operand (not used by a K-major one), 1024 bytes from one group of 8 rows to the next.
__device__ inline uint64_t operand(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(ATOM >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// code * scale of two (low and high half) pairs of codes, as two 16-bit pairs
__device__ inline uint2 widen(uint32_t codes, __half2 s1, __half2 s2) {
    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xffff), __NV_E4M3);
    const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> 16), __NV_E4M3);
    const __half2 x = __hmul2(__hmul2(__half2(a), s1), s2), y = __hmul2(__hmul2(__half2(b), s1), s2);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
}
__device__ inline uint2 widen(uint32_t codes, __nv_bfloat162 s1, __nv_bfloat162 s2) {
    // A code's 7 magnitude bits moved to bits 4..10 of a bf16 are the value times 2^-120, also
    // where it is subnormal; s1 is 2^120.
    uint32_t lo = __byte_perm(codes, 0, 0x1404), hi = __byte_perm(codes, 0, 0x3424);
    lo = (lo & 0x80008000u) | ((lo >> 4) & 0x07f007f0u);
    hi = (hi & 0x80008000u) | ((hi >> 4) & 0x07f007f0u);
    __nv_bfloat162 x = __hmul2(__hmul2(*reinterpret_cast<__nv_bfloat162 *>(&lo), s1), s2);
    __nv_bfloat162 y = __hmul2(__hmul2(*reinterpret_cast<__nv_bfloat162 *>(&hi), s1), s2);
    uint2 r = make_uint2(*reinterpret_cast<uint32_t *>(&x), *reinterpret_cast<uint32_t *>(&y));
    if (((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) {        // a NaN code among the four
        if ((codes & 0x7fu) == 0x7fu) r.x |= 0x7fffu;
        if ((codes & 0x7f00u) == 0x7f00u) r.x |= 0x7fff0000u;
        if ((codes & 0x7f0000u) == 0x7f0000u) r.y |= 0x7fffu;
        if ((codes & 0x7f000000u) == 0x7f000000u) r.y |= 0x7fff0000u;
    }
    return r;
}
// A scale as the two factors that widen() multiplies by.  f16: half the scale, so that nothing
// that came from f16 overflows, with a second factor for scales below the type's normal range.
__device__ inline void factors(float s, __half2 &s1, __half2 &s2) {
    s *= 0.5f;
    const float low = fabsf(s) < 6.103515625e-05f ? 5.9604644775390625e-08f : 1.0f;
    s1 = __float2half2_rn(s / low);
    s2 = __float2half2_rn(low);
}
__device__ inline void factors(float s, __nv_bfloat162 &s1, __nv_bfloat162 &s2) {
    s1 = __float2bfloat162_rn(1.329227995784916e+36f);                 // 2^120
    s2 = __float2bfloat162_rn(s);
}

template <typename T, bool C8, int D>
struct Many {
    static constexpr uint32_t KV = ATOM * (D / 64);         // bytes of a 128-row tile
    static constexpr uint32_t OFF_RING = 2 * KV;            // behind the two halves of Q
    static constexpr uint32_t OFF_BAR = OFF_RING + RING * KV;
    static constexpr uint32_t OFF_EXISTS = OFF_BAR + 256;   // [8 units][4]: keys that exist
    static constexpr uint32_t OFF_MISC = OFF_EXISTS + 128;
    static constexpr uint32_t SMEM = OFF_MISC + 256 + 1024; // 1024: alignment of the dynamic part
    // f16 codes are widened at half their value: scores and outputs make up for it
    static constexpr float VALUE = C8 && std::is_same<T, __half>::value ? 2.0f : 1.0f;
    // f16 probabilities are kept 2^6 times too large (at most 2^14): full precision down to 2^-20
    static constexpr float OFF = std::is_same<T, __half>::value ? 6.0f : 0.0f;
    using Pair = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    // byte offset of 16-byte chunk `ch` of row `row` in a tile
    __device__ static uint32_t place(uint32_t row, uint32_t ch) {
        return (ch >> 3) * ATOM + row * 128 + (((ch ^ row) & 7) << 4);
    }
};

template <typename T, bool C8, int D>
__global__ void __launch_bounds__(THREADS, 1) attend_many_kernel(const __grid_constant__ AttendParams p, const Workspace ws) {
    using C = Many<T, C8, D>;
    extern __shared__ unsigned char raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    unsigned char *sm = raw + (base - smem_addr(raw));
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    uint32_t *misc = reinterpret_cast<uint32_t *>(sm + C::OFF_MISC);
    uint32_t *exists = reinterpret_cast<uint32_t *>(sm + C::OFF_EXISTS);
    volatile uint32_t *dead = misc + 60;
    const uint32_t bars = base + C::OFF_BAR;
    const uint32_t full = bars, empty = bars + 32, q_full = bars + 64, q_empty = bars + 72, s_full = bars + 80,
                   p_full = bars + 96, o_full = bars + 112, o_empty = bars + 128, joined = bars + 144, drain = bars + 160;

    // ---- this worker's share ----
    unsigned long long *sums = reinterpret_cast<unsigned long long *>(misc);
    const uint32_t per = (p.step.n_seq + THREADS - 1) / THREADS;
    const uint32_t s_lo = threadIdx.x * per, s_hi = min(s_lo + per, p.step.n_seq);
    unsigned long long mine = 0;
    for (uint32_t s = s_lo; s < s_hi; ++s) {
        Tile t;
        const int code = tile_seq(p, s, t);
        if (code != TUTTI_OK && blockIdx.x == 0) report(p.step, code);
        mine += t.r.before(t.r.n_tiles) * p.pool.n_kv_heads;
    }
    unsigned long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    unsigned long long total = 0, start = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i < (int)warp) start += sums[i];
        total += sums[i];
    }
    start += incl - mine;
    const unsigned long long workers = total < ws.workers ? total : ws.workers;
    const uint32_t w = blockIdx.x;
    if (w >= workers) return;
    const unsigned long long x0 = w * total / workers, x1 = (w + 1) * total / workers;
    if (x0 >= start && x0 < start + mine) {
        unsigned long long at = start;
        for (uint32_t s = s_lo; s < s_hi; ++s) {
            Tile t;
            tile_seq(p, s, t);
            const unsigned long long n = t.r.before(t.r.n_tiles) * p.pool.n_kv_heads;
            if (x0 < at + n) {
                misc[32] = s;
                sums[14] = x0 - at;
                break;
            }
            at += n;
        }
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < RING; ++i) {
            mbar_init(full + 8 * i, PROD_WARPS);
            mbar_init(empty + 8 * i, 1);
        }
        mbar_init(q_full, PROD_WARPS);
        mbar_init(q_empty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 4);
            mbar_init(o_full + 8 * i, 1);
            mbar_init(o_empty + 8 * i, 4);
            mbar_init(joined + 8 * i, 4);
        }
        mbar_init(drain, 1);
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(base + C::OFF_MISC + 61 * 4) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_before();
    }
    __syncthreads();
    tc_after();
    const uint32_t tmem = misc[61];
    Tile t;
    tile_seq(p, misc[32], t);
    {
        const unsigned long long in_seq = sums[14], head = t.r.before(t.r.n_tiles);
        t.h = (uint32_t)(in_seq / head);
        const unsigned long long rest = in_seq % head;
        const Rows r = t.r;
        uint32_t lo = 0, len = r.n_tiles;               // last tile that starts at or before `rest`, 32 probes a round
        while (len > 1) {
            const uint32_t step = (len + 31) / 32;
            const bool le = lane * step < len && r.before(lo + lane * step) <= rest;
            const uint32_t last = 31 - __clz(__ballot_sync(0xffffffffu, le) | 1u);
            lo += last * step;
            len = min(len - last * step, step);
        }
        t.q = lo;
        t.u = (uint32_t)(rest - r.before(lo));
        t.n_units = r.units(lo);
    }
    // scores (and probabilities over them) of the halves, then their outputs
    auto S = [&](int i) { return tmem + i * 128; };
    auto O = [&](int i) { return tmem + 256 + i * D; };

    // Registers: 384 x 168 at launch = 256 x 192 + 128 x 120; a softmax thread holds its row's 128 scores.
    if (warp >= MMA_WARP) {
        setmaxnreg_dec<120>();
        if (warp >= PROD_WARP) {
        // =================================== gathering ===================================
        const uint32_t pw = warp - PROD_WARP;
        uint32_t n_put = 0, n_sig = 0, q_at = ~0u, segs = 0, n_unit = 0;
        bool ok = true;
        int64_t off[4];                                 // rows lane, lane + 32, ...: block id, -1 behind the end, -2 outside the pool
        float ks[4], vs[4];
        Tile f = t;                                     // the unit whose block ids are being looked up
        unsigned long long fx = x0;
        auto locate = [&]() {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t key = f.u * BN + i * 32 + lane;
                off[i] = -1;
                if (fx < x1 && key < f.v.ctx) {
                    const int32_t id = __ldg(p.step.block_ids + f.v.b0 + key / p.pool.block_tokens);
                    off[i] = (uint32_t)id < p.pool.n_blocks ? (int64_t)id : -2;
                }
            }
        };
        auto resolve = [&]() {                          // ids to byte offsets, scales; writes down which keys exist
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t key = f.u * BN + i * 32 + lane;
                if (off[i] == -2 && pw == 0) report(p.step, TUTTI_EFAULT);
                const bool there = off[i] >= 0;
                const uint32_t mask = __ballot_sync(0xffffffffu, off[i] != -2);   // keys behind the end are masked by position
                if (pw == 0 && lane == 0) exists[(n_unit & 7) * 4 + i] = mask;
                if (C8) {
                    const uint64_t at = there ? (uint64_t)off[i] * p.pool.n_kv_heads + f.h : 0;
                    ks[i] = there ? p.pool.k_scale[at] : 0.0f;
                    vs[i] = there ? p.pool.v_scale[at] : 0.0f;
                }
                if (there) off[i] = block_offset(p.pool, (int32_t)off[i]) + (int64_t)(key % p.pool.block_tokens * p.pool.tok_stride + f.h * p.pool.head_stride);
            }
            ++n_unit;
        };
        auto step_unit = [&]() {
            ++fx;
            if (fx < x1 && ++f.u == f.n_units) next_tile(p, f);
        };
        auto signal = [&](uint32_t upto) {              // tiles [n_sig, upto) have landed
            while (n_sig < upto) {
                fence_async();
                __syncwarp();
                if (lane == 0) {
                    if (n_sig == q_at) mbar_arrive(q_full);
                    mbar_arrive(full + 8 * (n_sig % RING));
                }
                ++n_sig;
            }
        };
        auto room = [&]() { return n_put < RING || mbar_wait(empty + 8 * (n_put % RING), (n_put / RING - 1) & 1, dead); };
        auto load_q = [&]() {                           // cp.async of the tile's rows, zeros behind the last
            constexpr int CH = D / 8;
            for (uint32_t i = pw; i < TILE_ROWS * CH / 32; i += PROD_WARPS) {
                const uint32_t r = (i * 32 + lane) / CH, ch = lane % CH, row = t.q * TILE_ROWS + r;
                const bool in = row < t.r.n_rows;
                const uint32_t n = in ? row / p.group : 0, h = t.h * p.group + (in ? row % p.group : 0);
                const T *src = (const T *)p.q + (uint64_t)(t.v.q0 + n) * p.q_stride + (uint64_t)h * D + ch * 8;
                cp16(base + r / HALF_ROWS * C::KV + C::place(r % HALF_ROWS, ch), src, in);
            }
        };
        constexpr int CH = D * (C8 ? 1 : 2) / 16;       // 16-byte chunks of a row in the pool
        constexpr int RPI = 32 / CH;                    // rows a warp takes at once
        constexpr int PER = 32 / RPI;                   // such steps in 32 rows
        constexpr int N = (PER + PROD_WARPS - 1) / PROD_WARPS;
        const uint32_t ch = lane % CH, sub = lane / CH;
        locate();
        uint4 rk[C8 ? 4 : 1][C8 ? N : 1], rv[C8 ? 4 : 1][C8 ? N : 1];
        float cs[4];
        auto fetch8 = [&](uint4 (&r)[C8 ? 4 : 1][C8 ? N : 1], uint64_t from) {
            if constexpr (C8) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const uint32_t it = (pw + i) % PROD_WARPS + PROD_WARPS * k;
                        r[i][k] = make_uint4(0, 0, 0, 0);
                        if (it < PER) {
                            const int64_t o = __shfl_sync(0xffffffffu, off[i], it * RPI + sub);
                            if (o >= 0) r[i][k] = __ldg(reinterpret_cast<const uint4 *>(from + o + ch * 16));
                        }
                    }
            }
        };
        auto store8 = [&](const uint4 (&r)[C8 ? 4 : 1][C8 ? N : 1], const float (&sc)[4], uint32_t slot) {
            if constexpr (C8) {
                const uint32_t dst = C::OFF_RING + slot * C::KV;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const uint32_t it = (pw + i) % PROD_WARPS + PROD_WARPS * k;
                        if (it < PER) {
                            const uint32_t row = i * 32 + it * RPI + sub;
                            typename C::Pair s1, s2;
                            factors(__shfl_sync(0xffffffffu, sc[i], it * RPI + sub), s1, s2);
                            const uint2 a = widen(r[i][k].x, s1, s2), b = widen(r[i][k].y, s1, s2);
                            const uint2 c = widen(r[i][k].z, s1, s2), d = widen(r[i][k].w, s1, s2);
                            *reinterpret_cast<uint4 *>(sm + dst + C::place(row, 2 * ch)) = make_uint4(a.x, a.y, b.x, b.y);
                            *reinterpret_cast<uint4 *>(sm + dst + C::place(row, 2 * ch + 1)) = make_uint4(c.x, c.y, d.x, d.y);
                        }
                    }
            }
        };
        if constexpr (C8) {
            resolve();
            fetch8(rk, p.pool.k_base);
        }
        for (unsigned long long x = x0; x < x1 && ok;) {
            const uint32_t n = (uint32_t)min(x1 - x, (unsigned long long)(t.n_units - t.u));
            if (segs) {
                cp_wait<0>();
                signal(n_put);
                ok = mbar_wait(q_empty, (segs - 1) & 1, dead);
                if (!ok) break;
            }
            load_q();
            if constexpr (C8) {
                cp_commit();
                cp_wait<0>();
                fence_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full);
            } else {
                q_at = n_put;
            }
            for (uint32_t j = 0; j < n && ok; ++j) {
                if constexpr (!C8) {
                    resolve();
                    for (int half = 0; half < 2 && ok; ++half) {
                        ok = room();
                        if (!ok) break;
                        const uint32_t dst = base + C::OFF_RING + (n_put % RING) * C::KV;
                        const uint64_t from = half ? p.pool.v_base : p.pool.k_base;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int k = 0; k < N; ++k) {
                                const uint32_t it = (pw + i) % PROD_WARPS + PROD_WARPS * k;
                                if (it < PER) {
                                    const uint32_t row = it * RPI + sub;
                                    const int64_t o = __shfl_sync(0xffffffffu, off[i], row);
                                    cp16(dst + C::place(i * 32 + row, ch), (const void *)(from + (o >= 0 ? o : 0) + ch * 16), o >= 0);
                                }
                            }
                        cp_commit();
                        ++n_put;
                        cp_wait<2>();
                        if (n_put >= 2) signal(n_put - 2);
                    }
                    step_unit();
                    locate();
                } else {
                    fetch8(rv, p.pool.v_base);
                    ok = room();
                    if (!ok) break;
                    store8(rk, ks, n_put % RING);
                    ++n_put;
                    signal(n_put);
#pragma unroll
                    for (int i = 0; i < 4; ++i) cs[i] = vs[i];
                    step_unit();
                    locate();
                    if (fx < x1) {
                        resolve();
                        fetch8(rk, p.pool.k_base);
                    }
                    ok = room();
                    if (!ok) break;
                    store8(rv, cs, n_put % RING);
                    ++n_put;
                    signal(n_put);
                }
            }
            x += n;
            ++segs;
            if (x < x1) next_tile(p, t);
        }
        cp_wait<0>();
        if (ok) signal(n_put);
        } else {
        // =================================== matrix instructions ===================================
        if (lane == 0) {
            constexpr uint32_t FMT = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
            constexpr uint32_t IDESC = 1u << 4 | FMT << 7 | FMT << 10 | (uint32_t)(HALF_ROWS / 16) << 24;
            constexpr uint32_t ID_QK = IDESC | (uint32_t)(BN / 8) << 17, ID_PV = IDESC | 1u << 16 | (uint32_t)(D / 8) << 17;
            uint32_t kv = 0, segs = 0, np[2] = {0, 0}, ns[2] = {0, 0};
            bool ok = true;
            auto qk = [&](int i, uint32_t slot) {
                const uint64_t a = operand(base + i * C::KV), b = operand(base + C::OFF_RING + slot * C::KV);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint64_t step = ((k / 4) * ATOM + (k % 4) * 32) >> 4;
                    mma_ss(S(i), a + step, b + step, ID_QK, k > 0);
                }
                tc_commit(s_full + 8 * i);
            };
            auto pv = [&](int i, uint32_t slot, bool acc) {
                const uint64_t b = operand(base + C::OFF_RING + slot * C::KV);
#pragma unroll
                for (int k = 0; k < BN / 16; ++k) mma_ts(O(i), S(i) + k * 8, b + ((k * 2048) >> 4), ID_PV, acc || k > 0);
                tc_commit(o_full + 8 * i);
            };
            auto landed = [&](uint32_t i) { return mbar_wait(full + 8 * (i % RING), (i / RING) & 1, dead); };
            for (unsigned long long x = x0; x < x1 && ok;) {
                const uint32_t n = (uint32_t)min(x1 - x, (unsigned long long)(t.n_units - t.u));
                const int halves = t.r.n_rows - t.q * TILE_ROWS > HALF_ROWS ? 2 : 1;
                ok = mbar_wait(q_full, segs & 1, dead) && landed(kv);
                if (!ok) break;
                tc_after();
                for (int i = 0; i < halves; ++i) qk(i, kv % RING);
                tc_commit(empty + 8 * (kv % RING));
                ++kv;
                for (uint32_t j = 0; j < n && ok; ++j) {
                    const bool more = j + 1 < n;
                    ok = landed(kv) && (!more || landed(kv + 1));
                    for (int i = 0; i < halves && ok; ++i) {
                        ok = mbar_wait(p_full + 8 * i, np[i]++ & 1, dead);
                        if (ok && j == 0 && ns[i]) ok = mbar_wait(o_empty + 8 * i, (ns[i] - 1) & 1, dead);
                        if (!ok) break;
                        tc_after();
                        pv(i, kv % RING, j > 0);
                        if (more) qk(i, (kv + 1) % RING);
                    }
                    if (!ok) break;
                    tc_commit(empty + 8 * (kv % RING));
                    if (more) tc_commit(empty + 8 * ((kv + 1) % RING));
                    kv += more ? 2 : 1;
                }
                if (!ok) break;
                for (int i = 0; i < halves; ++i) ++ns[i];
                tc_commit(q_empty);
                ++segs;
                x += n;
                if (x < x1) next_tile(p, t);
            }
            // every matrix instruction has ended before TMEM is given back
            tc_commit(drain);
            const long long t0 = clock64();
            while (!mbar_try(drain, 0) && clock64() - t0 < WAIT_CLOCKS) {}
        }
        __syncwarp();
        }
    } else {
        // =================================== softmax ===================================
        setmaxnreg_inc<192>();
        const int i = warp / 4;                                   // half
        const uint32_t lanes = (warp % 4) * 32 << 16, s_at = S(i) + lanes, o_at = O(i) + lanes, r = (warp % 4) * 32 + lane;
        const float scl = fmaxf(fabsf(p.scale) * 1.4426950408889634f * C::VALUE, 1e-30f);
        const bool negative = p.scale < 0;
        uint32_t n_s = 0, n_unit = 0, n_join = 0;                 // scores seen by this half; units of the worker
        bool ok = true;
        auto join = [&]() {                                       // the half's four warps
            __syncwarp();
            if (lane == 0) mbar_arrive(joined + 8 * i);
            const bool there = mbar_wait(joined + 8 * i, n_join++ & 1, dead);
            return (bool)__all_sync(0xffffffffu, there);
        };
        for (unsigned long long x = x0; x < x1 && ok;) {
            const uint32_t n = (uint32_t)min(x1 - x, (unsigned long long)(t.n_units - t.u));
            const uint32_t row = t.q * TILE_ROWS + i * HALF_ROWS + r;
            if (t.q * TILE_ROWS + i * HALF_ROWS < t.r.n_rows) {
                const bool in = row < t.r.n_rows;
                // rows behind the last take the last one's position: they are computed and dropped
                const uint32_t tok = (in ? row : t.r.n_rows - 1) / p.group;
                const int64_t pos = t.r.first + tok;
                const int64_t pos_low = __shfl_sync(0xffffffffu, pos, 0);
                float m = -INFINITY, l = 0;
                for (uint32_t j = 0; j < n && ok; ++j) {
                    ok = mbar_wait(s_full + 8 * i, n_s & 1, dead);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_after();
                    uint32_t sr[128];
                    float *s = reinterpret_cast<float *>(sr);
#pragma unroll
                    for (int q = 0; q < 4; ++q) tc_ld32(sr + 32 * q, s_at + 32 * q);
                    const uint4 ex = *reinterpret_cast<const uint4 *>(exists + ((n_unit + j) & 7) * 4);
                    tc_wait_ld();
#pragma unroll
                    for (int q = 0; q < 4; ++q) tc_loaded(sr + 32 * q);
                    const int64_t key0 = (int64_t)(t.u + j) * BN;
                    if (negative) {
#pragma unroll
                        for (int k = 0; k < 128; ++k) s[k] = -s[k];
                    }
                    if (key0 + BN - 1 > pos_low || (ex.x & ex.y & ex.z & ex.w) != ~0u) {
                        const int64_t d = pos - key0;
                        const int lim = d < -1 ? -1 : d > BN ? BN : (int)d;
                        const uint32_t word[4] = {ex.x, ex.y, ex.z, ex.w};
#pragma unroll
                        for (int k = 0; k < 128; ++k)
                            if (k > lim || !(word[k / 32] >> (k % 32) & 1)) s[k] = -INFINITY;
                    }
                    float a0 = s[0], a1 = s[1], a2 = s[2], a3 = s[3];
#pragma unroll
                    for (int k = 4; k < 128; k += 4) {
                        a0 = fmaxf(a0, s[k]);
                        a1 = fmaxf(a1, s[k + 1]);
                        a2 = fmaxf(a2, s[k + 2]);
                        a3 = fmaxf(a3, s[k + 3]);
                    }
                    const float top = fmaxf(fmaxf(a0, a1), fmaxf(a2, a3)) * scl;
                    const bool grow = top > m + GROW || (m == -INFINITY && top > m);
                    if (__any_sync(0xffffffffu, grow)) {
                        const float alpha = grow ? ex2(m - top) : 1.0f;
                        if (grow) m = top;
                        l *= alpha;
                        if (j > 0) {
                            ok = mbar_wait(o_full + 8 * i, (n_s - 1) & 1, dead);
                            ok = __all_sync(0xffffffffu, ok);
                            if (!ok) break;
                            tc_after();
#pragma unroll
                            for (int q = 0; q < D / 32; ++q) {
                                uint32_t o[32];
                                tc_ld32(o, o_at + 32 * q);
                                tc_wait_ld();
                                tc_loaded(o);
#pragma unroll
                                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                                tc_st32(o, o_at + 32 * q);
                            }
                        }
                    }
                    const float sub = (m == -INFINITY ? 0.0f : m) - C::OFF;
                    float l0 = 0, l1 = 0, l2 = 0, l3 = 0;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t pk[16];
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float e0 = ex2(fmaf(s[32 * q + k], scl, -sub)), e1 = ex2(fmaf(s[32 * q + k + 1], scl, -sub));
                            const float e2 = ex2(fmaf(s[32 * q + k + 2], scl, -sub)), e3 = ex2(fmaf(s[32 * q + k + 3], scl, -sub));
                            l0 += e0, l1 += e1, l2 += e2, l3 += e3;
                            pk[k / 2] = pack2(e0, e1, T());
                            pk[k / 2 + 1] = pack2(e2, e3, T());
                        }
                        tc_st16(pk, s_at + 16 * q);
                    }
                    l += (l0 + l1) + (l2 + l3);
                    tc_wait_st();
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 8 * i);
                    ++n_s;
                }
                if (!ok) break;
                ok = mbar_wait(o_full + 8 * i, (n_s - 1) & 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_after();
                bool write = true;
                const bool whole = t.u == 0 && n == t.n_units;
                float o[D];
#pragma unroll
                for (int q = 0; q < D / 32; ++q) tc_ld32(reinterpret_cast<uint32_t *>(o) + 32 * q, o_at + 32 * q);
                tc_wait_ld();
#pragma unroll
                for (int q = 0; q < D / 32; ++q) tc_loaded(reinterpret_cast<uint32_t *>(o) + 32 * q);
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_empty + 8 * i);
                if (!whole) {
                    const unsigned long long tile0 = x - t.u;
                    const uint32_t w0 = (uint32_t)(((tile0 + 1) * workers - 1) / total);
                    const uint32_t w1 = (uint32_t)(((tile0 + t.n_units) * workers - 1) / total);
                    auto slot = [&](uint32_t k) { return (k == w0 ? 2 * k + 1 : 2 * k) * 2 + i; };
                    float4 *part = reinterpret_cast<float4 *>(ws.part);
                    float2 *ml = reinterpret_cast<float2 *>(ws.part + (uint64_t)4 * ws.workers * HALF_ROWS * D);
                    auto at = [&](uint32_t k, int d4) { return part + ((uint64_t)slot(k) * (D / 4) + d4) * HALF_ROWS + r; };
#pragma unroll
                    for (int d = 0; d < D / 4; ++d) *at(w, d) = make_float4(o[4 * d], o[4 * d + 1], o[4 * d + 2], o[4 * d + 3]);
                    ml[(uint64_t)slot(w) * HALF_ROWS + r] = make_float2(m, l);
                    __threadfence();
                    if (!(ok = join())) break;
                    if (r == 0) {
                        const uint32_t old = atomicAdd(ws.count + 2 * w0 + i, 1);
                        if (old == w1 - w0) ws.count[2 * w0 + i] = 0;            // ready for the next call
                        misc[40 + i] = old == w1 - w0;
                    }
                    if (!(ok = join())) break;
                    write = *(volatile uint32_t *)(misc + 40 + i);
                    if (write) {
                        __threadfence();
                        m = -INFINITY;
                        l = 0;
                        for (uint32_t k = w0; k <= w1; ++k) m = fmaxf(m, __ldcg(ml + (uint64_t)slot(k) * HALF_ROWS + r).x);
#pragma unroll
                        for (int d = 0; d < D; ++d) o[d] = 0;
                        for (uint32_t k = w0; k <= w1; ++k) {
                            const float2 e = __ldcg(ml + (uint64_t)slot(k) * HALF_ROWS + r);
                            const float c = m == -INFINITY ? 0.0f : ex2(e.x - m);
                            l += e.y * c;
#pragma unroll
                            for (int d = 0; d < D / 4; ++d) {
                                const float4 b = __ldcg(at(k, d));
                                o[4 * d] += b.x * c, o[4 * d + 1] += b.y * c, o[4 * d + 2] += b.z * c, o[4 * d + 3] += b.w * c;
                            }
                        }
                    }
                }
                if (write && in) {
                    const uint64_t token = t.v.q0 + tok;
                    const uint32_t qh = t.h * p.group + row % p.group;
                    const float inv = m == -INFINITY ? 0.0f : C::VALUE / l;
                    uint4 *out = reinterpret_cast<uint4 *>((T *)p.out + token * p.out_stride + (uint64_t)qh * D);
#pragma unroll
                    for (int d = 0; d < D / 8; ++d)
                        out[d] = make_uint4(pack2(o[8 * d] * inv, o[8 * d + 1] * inv, T()), pack2(o[8 * d + 2] * inv, o[8 * d + 3] * inv, T()),
                                            pack2(o[8 * d + 4] * inv, o[8 * d + 5] * inv, T()), pack2(o[8 * d + 6] * inv, o[8 * d + 7] * inv, T()));
                    if (p.lse) p.lse[token * p.n_q_heads + qh] = m == -INFINITY ? -INFINITY : (m - C::OFF + log2f(l)) * 0.6931471805599453f;
                }
            }
            n_unit += n;
            x += n;
            if (x < x1) next_tile(p, t);
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (threadIdx.x == 0 && *dead) report(p.step, TUTTI_ETIMEDOUT);
    if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <typename T, bool C8, int D>
cudaError_t launch(const AttendParams &p, const Workspace &ws, cudaStream_t st) {
    attend_many_kernel<T, C8, D><<<ws.workers, THREADS, Many<T, C8, D>::SMEM, st>>>(p, ws);
    return cudaGetLastError();
}

template <typename T, bool C8>
cudaError_t launch(const AttendParams &p, const Workspace &ws, cudaStream_t st) {
    return p.pool.head_dim == 128 ? launch<T, C8, 128>(p, ws, st) : launch<T, C8, 64>(p, ws, st);
}

template <typename T, bool C8, int D>
cudaError_t setup() {
    return cudaFuncSetAttribute(attend_many_kernel<T, C8, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Many<T, C8, D>::SMEM);
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

cudaError_t many_launch(const AttendParams &p, const Workspace &ws, bool c8, bool bf, cudaStream_t st) {
    if (c8) return bf ? launch<__nv_bfloat16, true>(p, ws, st) : launch<__half, true>(p, ws, st);
    return bf ? launch<__nv_bfloat16, false>(p, ws, st) : launch<__half, false>(p, ws, st);
}

uint32_t many_workers(int sms) { return (uint32_t)sms; }
size_t many_part_bytes(uint32_t workers) { return (size_t)4 * workers * HALF_ROWS * (128 + 2) * sizeof(float); }

}  // namespace tutti

// The kernel's own count of units, on the host: out2[0] units of tile q, out2[1] units of the tiles before it.
extern "C" int tutti_many_units_(uint32_t ctx, uint32_t n_new, uint32_t group, uint32_t q, uint64_t *out2) {
    const tutti::SeqView v{0, n_new, ctx, 0};
    const tutti::Rows r = tutti::rows_of(v, group);
    out2[0] = q < r.n_tiles ? r.units(q) : 0;
    out2[1] = r.before(q);
    return (int)r.n_tiles;
}
