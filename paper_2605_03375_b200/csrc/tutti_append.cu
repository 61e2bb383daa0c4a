// Appending a step's keys and values to a layer of the paged pool, with the position rotation of
// queries and keys applied on the way:
//     y1 = x1 cos - x2 sin,  y2 = x2 cos + x1 sin      for every pair (x1, x2) that turns together
// in 32 bits, rounded once.  In an 8-bit pool a key or value is stored as rn_e4m3(x / s), s the
// power of two of its block and head.
//
// The unit of both kernels is a *job*: the 16 elements of one head's row that one thread loads
// as two 16-byte vectors, chosen so that every pair is inside one job (half-split style: the
// vectors at d and d + rot_dim / 2).  head_dim / 16 lanes cover a row, a warp 32 / (head_dim / 16)
// rows at a time.  Every input is read once and every output written once; the bound is HBM
// bandwidth for prompts and latency for a decode step: the search of the sequence, its tables, the
// block's id and the rows are loads that wait for each other.
// On a B200 (6.45 TB/s copy): 16384 tokens of 48 rows of 128, bf16, 72 us = 5.7 TB/s; 12187 tokens of
// 80 rows, fp16, into an 8-bit pool 107 us = 4.5 TB/s (blocks of 32 or 64 tokens, read twice: 114 and 115); 64 single tokens 4.0 and 6.6 us.  24 warps an SM
// (80 registers, a few spilled) against 16: 72 against 75 us, 106 against 109; 32: 92 us.
#include <cuda_fp8.h>

#include "tutti_paged.h"

namespace tutti {

namespace {

constexpr int THREADS = 256;
// Once a step has more rows than this, which fill the GPU's warps, a warp takes all rows of its
// token (up to PASSES x (32 / jobs) of them): finding the sequence and the block costs it as much as
// moving a few rows (16384 tokens of 48 rows: 169 us at 2 passes a warp, 108 at 4, 97 at 8, 76 at
// 12, all of them).  Below, one pass, for latency.
constexpr uint64_t ROWS_ENOUGH = 32768;
constexpr uint32_t PASSES = 16;
constexpr int SCALE_MIN_EXP = -100;     // never zero: dividing by a scale is exact and finite

struct RopeDev {
    uint32_t rot_dim;       // 0: nothing turns
    uint32_t pairs;
    uint32_t n_pos;
    const float *table;
};

struct AppendParams {
    StepDev step;
    PoolView pool;
    RopeDev rope;
    uint32_t n_q_heads;
    uint64_t q_stride, k_stride, v_stride, q_out_stride;   // bytes
    const char *q, *k, *v;
    char *q_out;
    uint32_t jobs;          // head_dim / 16
    uint32_t row_passes;    // rows_per_pass rows are taken this many times by a warp
    uint32_t row_units;     // warps per token of the row part
    uint32_t n_row_warps;   // n_tok * row_units
    uint32_t blk_units;     // touched-block slots (8-bit pool)
};

__device__ inline float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ inline float to_f(__half x) { return __half2float(x); }

template <typename T>
__device__ inline void unpack(const uint4 &u, float *x) {
    const T *e = reinterpret_cast<const T *>(&u);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f(e[i]);
}

template <typename T>
__device__ inline uint4 pack(const float *x) {
    return make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()), pack2(x[6], x[7], T()));
}

// Elements of job j of a row: the two vectors start at d0 and d1; `turn` says whether they rotate
// and t0 which cosine (and sine) is the first of the eight they need.
struct Job {
    uint32_t d0, d1, t0;
    bool turn;
};

__device__ inline Job job_of(const RopeDev &r, uint32_t j) {
    Job b;
    if (r.pairs || 16 * j >= r.rot_dim) {
        b.d0 = 16 * j;
        b.d1 = b.d0 + 8;
        b.t0 = 8 * j;
        b.turn = b.d0 < r.rot_dim;
    } else {
        b.d0 = b.t0 = 8 * j;
        b.d1 = b.d0 + r.rot_dim / 2;
        b.turn = true;
    }
    return b;
}

struct Turn {
    float c[8], s[8];
};

__device__ inline void load_turn(const RopeDev &r, uint32_t pos, uint32_t t0, Turn &t) {
    const float4 *p = reinterpret_cast<const float4 *>(r.table + (uint64_t)pos * r.rot_dim + t0);
    const float4 *s = reinterpret_cast<const float4 *>(r.table + (uint64_t)pos * r.rot_dim + r.rot_dim / 2 + t0);
    *reinterpret_cast<float4 *>(t.c) = __ldg(p);
    *reinterpret_cast<float4 *>(t.c + 4) = __ldg(p + 1);
    *reinterpret_cast<float4 *>(t.s) = __ldg(s);
    *reinterpret_cast<float4 *>(t.s + 4) = __ldg(s + 1);
}

// x: the 16 elements of a job, in the order they were loaded
__device__ inline void rotate(const RopeDev &r, const Turn &t, float *x) {
    auto turn = [](float &a, float &b, float c, float s) {
        const float x1 = a, x2 = b;
        a = x1 * c - x2 * s;
        b = x2 * c + x1 * s;
    };
    if (r.pairs) {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn(x[2 * i], x[2 * i + 1], t.c[i], t.s[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn(x[i], x[8 + i], t.c[i], t.s[i]);
    }
}

// One token's rows [0, n_rows): queries, and with KV its keys and values behind them.
template <typename T, bool KV>
__device__ void row_warp(const AppendParams &p, uint32_t w) {
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t tok = w / p.row_units, unit = w % p.row_units;
    const uint32_t s = warp_find(p.step.n_seq, tok, [&](uint32_t i) { return __ldg(p.step.q_start + i); });
    if (tok >= __ldg(p.step.q_start + p.step.n_seq)) return;      // behind the last sequence
    SeqView v;
    int code = seq_view(p.step, p.pool.block_tokens, s, v);
    if (code == TUTTI_OK && s == 0 && tok < v.q0) return;         // before the first one
    if (code == TUTTI_OK && (tok < v.q0 || tok - v.q0 >= v.n_new)) code = TUTTI_EINVAL;
    if (code == TUTTI_OK && p.rope.rot_dim && v.ctx > p.rope.n_pos) code = TUTTI_EINVAL;
    if (code != TUTTI_OK) {
        if (lane == 0) report(p.step, code);
        return;
    }
    const int64_t pos = (int64_t)v.ctx - v.n_new + (tok - v.q0);
    if (pos < 0) return;
    int64_t at = 0;
    if (KV) {
        at = block_offset(p.pool, __ldg(p.step.block_ids + v.b0 + p.pool.block_of((uint32_t)pos)));
        if (at < 0) {
            if (lane == 0) report(p.step, TUTTI_EFAULT);
        } else {
            at += (int64_t)(p.pool.row_of((uint32_t)pos) * p.pool.tok_stride);
        }
    }
    const uint32_t per = 32 / p.jobs, j = lane % p.jobs;
    if (lane / p.jobs >= per) return;
    const Job b = job_of(p.rope, j);
    Turn t;
    if (b.turn) load_turn(p.rope, (uint32_t)pos, b.t0, t);
    const uint32_t hk = p.pool.n_kv_heads, hd = p.pool.head_dim;
    const uint32_t n_rows = p.n_q_heads + (KV ? 2 * hk : 0);
    const uint32_t first = unit * p.row_passes * per + lane / p.jobs;
    // Four rows' loads are issued before the first store: a store might alias a later load as far as
    // the compiler knows, and one row in flight at a time leaves the memory idle.
    for (uint32_t i0 = 0; i0 < p.row_passes; i0 += 4) {
        uint4 u[4][2];
        char *dst[4];
        bool turn[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = first + (i0 + i) * per;
            dst[i] = nullptr;
            if (i0 + i >= p.row_passes || r >= n_rows) continue;
            const char *src;
            turn[i] = b.turn;
            if (r < p.n_q_heads) {
                src = p.q + tok * p.q_stride + (uint64_t)r * hd * 2;
                dst[i] = p.q_out + tok * p.q_out_stride + (uint64_t)r * hd * 2;
            } else {
                if (at < 0) continue;
                const bool is_v = r >= p.n_q_heads + hk;
                const uint32_t h = r - p.n_q_heads - (is_v ? hk : 0);
                src = (is_v ? p.v + tok * p.v_stride : p.k + tok * p.k_stride) + (uint64_t)h * hd * 2;
                dst[i] = (char *)((is_v ? p.pool.v_base : p.pool.k_base) + at + h * p.pool.head_stride);
                turn[i] = b.turn && !is_v;
            }
            u[i][0] = *reinterpret_cast<const uint4 *>(src + b.d0 * 2);
            u[i][1] = *reinterpret_cast<const uint4 *>(src + b.d1 * 2);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!dst[i]) continue;
            if (turn[i]) {
                float x[16];
                unpack<T>(u[i][0], x);
                unpack<T>(u[i][1], x + 8);
                rotate(p.rope, t, x);
                u[i][0] = pack<T>(x);
                u[i][1] = pack<T>(x + 8);
            }
            *reinterpret_cast<uint4 *>(dst[i] + b.d0 * 2) = u[i][0];
            *reinterpret_cast<uint4 *>(dst[i] + b.d1 * 2) = u[i][1];
        }
    }
}

// Smallest power of two s with amax / s <= 448 = 1.75 * 2^8, by the bits of amax: its exponent less
// 8, one more where the mantissa is above 1.75.
__device__ inline float pow2_scale(float amax) {
    const int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 127 - 8;
    return __uint_as_float((uint32_t)(max(e, SCALE_MIN_EXP) + 127) << 23);
}

__device__ inline float finite_abs(float x) {
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.0f;       // infinities and NaN do not count
}

__device__ inline uint2 codes_of(const float *x, float inv) {
    uint32_t r[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __nv_fp8x2_storage_t a = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i] * inv, x[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        const __nv_fp8x2_storage_t b = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2] * inv, x[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
        r[i] = (uint32_t)a | (uint32_t)b << 16;
    }
    return make_uint2(r[0], r[1]);
}

// One touched block of one head, keys or values: the largest new value, the scale, the codes.
// The block's rows belong to this warp alone.
template <typename T>
__device__ void block_warp(const AppendParams &p, uint32_t w) {
    const uint32_t lane = threadIdx.x & 31, hk = p.pool.n_kv_heads, bs = p.pool.block_tokens;
    const uint32_t h = w % hk, is_v = w / hk % 2, u = w / hk / 2;
    // Slots of sequence s: [q_start[s] / bs + 2 s, q_start[s+1] / bs + 2 s + 2).  n rows touch at
    // most (n - 1) / bs + 2 blocks, so they fit, and no prefix sum over the sequences is needed.
    const uint32_t s = warp_find(p.step.n_seq, u, [&](uint32_t i) { return __ldg(p.step.q_start + i) / bs + 2 * i; });
    SeqView v;
    int code = seq_view(p.step, bs, s, v);
    if (code == TUTTI_OK && p.rope.rot_dim && v.ctx > p.rope.n_pos) code = TUTTI_EINVAL;
    if (code != TUTTI_OK) {
        if (lane == 0) report(p.step, code);
        return;
    }
    const uint32_t n_new = min(v.n_new, v.ctx);                  // the others are padding
    if (n_new == 0) return;
    const uint32_t first = v.ctx - n_new, row0 = v.q0 + v.n_new - n_new;
    const uint32_t blk = first / bs + (u - (v.q0 / bs + 2 * s));
    if (u < v.q0 / bs + 2 * s || (uint64_t)blk * bs >= v.ctx) return;
    const int32_t id = __ldg(p.step.block_ids + v.b0 + blk);
    const int64_t at = block_offset(p.pool, id);
    if (at < 0) {
        if (lane == 0) report(p.step, TUTTI_EFAULT);
        return;
    }
    const uint32_t lo = max(first, blk * bs), hi = min((uint64_t)v.ctx, ((uint64_t)blk + 1) * bs);
    char *rows = (char *)((is_v ? p.pool.v_base : p.pool.k_base) + at + h * p.pool.head_stride);
    float *scale = (is_v ? p.pool.v_scale : p.pool.k_scale) + (uint64_t)id * p.pool.scale_row + h;
    const uint64_t in_stride = is_v ? p.v_stride : p.k_stride;
    const char *in = (is_v ? p.v : p.k) + (uint64_t)h * p.pool.head_dim * 2;
    const uint32_t per = 32 / p.jobs, j = lane % p.jobs, sub = lane / p.jobs;
    const Job b = job_of(p.rope, j);
    const bool turn = b.turn && !is_v;

    // Up to HELD passes stay in registers between finding the largest value and writing the codes;
    // larger parts of a block are read twice (the second time out of L1/L2).
    constexpr uint32_t HELD = 4;
    const bool held_all = hi - lo <= HELD * per;
    uint4 raw[HELD][2];
    auto expand = [&](const uint4 (&v)[2], uint32_t pos, float *x) {
        unpack<T>(v[0], x);
        unpack<T>(v[1], x + 8);
        if (turn) {
            Turn t;
            load_turn(p.rope, pos, b.t0, t);
            rotate(p.rope, t, x);
        }
    };
    auto load = [&](uint32_t pos, float *x) {
        const char *src = in + (uint64_t)(row0 + (pos - first)) * in_stride;
        const uint4 v[2] = {*reinterpret_cast<const uint4 *>(src + b.d0 * 2), *reinterpret_cast<const uint4 *>(src + b.d1 * 2)};
        expand(v, pos, x);
    };
    // The block's earlier codes are fetched along: whether they have to be rounded again is known late.
    const uint32_t held = lo - blk * bs;
    const float old = held ? *scale : 0.0f;
    uint2 was[HELD][2];
    auto earlier = [&](uint32_t r, uint32_t c) { return reinterpret_cast<uint2 *>(rows + r * p.pool.tok_stride + (c ? b.d1 : b.d0)); };
#pragma unroll
    for (uint32_t i = 0; i < HELD; ++i) {
        const uint32_t r = sub + i * per;
        if (sub < per && r < held) {
            was[i][0] = *earlier(r, 0);
            was[i][1] = *earlier(r, 1);
        }
    }
    float amax = 0.0f;
    if (held_all) {
#pragma unroll
        for (uint32_t i = 0; i < HELD; ++i) {
            const uint32_t pos = lo + sub + i * per;
            if (sub < per && pos < hi) {
                const char *src = in + (uint64_t)(row0 + (pos - first)) * in_stride;
                raw[i][0] = *reinterpret_cast<const uint4 *>(src + b.d0 * 2);
                raw[i][1] = *reinterpret_cast<const uint4 *>(src + b.d1 * 2);
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < HELD; ++i) {
            const uint32_t pos = lo + sub + i * per;
            if (sub < per && pos < hi) {
                float x[16];
                expand(raw[i], pos, x);
#pragma unroll
                for (int k = 0; k < 16; ++k) amax = fmaxf(amax, finite_abs(x[k]));
            }
        }
    } else if (sub < per) {
        for (uint32_t pos = lo + sub; pos < hi; pos += per) {
            float x[16];
            load(pos, x);
#pragma unroll
            for (int i = 0; i < 16; ++i) amax = fmaxf(amax, finite_abs(x[i]));
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    float sc = pow2_scale(amax);
    if (held) {
        sc = fmaxf(sc, old);
        if (sc != old && sub < per) {
            const float ratio = old / sc;
            auto again = [&](const uint2 &codes) {
                const __nv_fp8_e4m3 *e = reinterpret_cast<const __nv_fp8_e4m3 *>(&codes);
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (float)e[i];
                return codes_of(x, ratio);
            };
#pragma unroll
            for (uint32_t i = 0; i < HELD; ++i) {
                const uint32_t r = sub + i * per;
                if (r < held) {
                    *earlier(r, 0) = again(was[i][0]);
                    *earlier(r, 1) = again(was[i][1]);
                }
            }
            for (uint32_t r = sub + HELD * per; r < held; r += per) {
                *earlier(r, 0) = again(*earlier(r, 0));
                *earlier(r, 1) = again(*earlier(r, 1));
            }
        }
    }
    const float inv = 1.0f / sc;          // exact: a power of two
    auto write = [&](uint32_t pos, const float *x) {
        char *dst = rows + (pos - blk * bs) * p.pool.tok_stride;
        *reinterpret_cast<uint2 *>(dst + b.d0) = codes_of(x, inv);
        *reinterpret_cast<uint2 *>(dst + b.d1) = codes_of(x + 8, inv);
    };
    if (held_all) {
#pragma unroll
        for (uint32_t i = 0; i < HELD; ++i) {
            const uint32_t pos = lo + sub + i * per;
            if (sub < per && pos < hi) {
                float x[16];
                expand(raw[i], pos, x);
                write(pos, x);
            }
        }
    } else if (sub < per) {
        for (uint32_t pos = lo + sub; pos < hi; pos += per) {
            float x[16];
            load(pos, x);
            write(pos, x);
        }
    }
    __syncwarp();                         // every lane has read the old scale
    if (lane == 0) *scale = sc;
}

template <typename T>
__global__ void __launch_bounds__(THREADS, 3) append_kernel(const __grid_constant__ AppendParams p) {
    const uint32_t w = (blockIdx.x * (uint64_t)THREADS + threadIdx.x) / 32;
    if (w < p.n_row_warps) row_warp<T, true>(p, w);
    // A copy kernel behind this one in the stream may be launched as soon as every CTA has ended
    // (it is a programmatic dependent): what was written must be visible by then.
    __threadfence();
}

template <typename T>
__global__ void __launch_bounds__(THREADS, 3) append8_kernel(const __grid_constant__ AppendParams p) {
    const uint32_t w = (blockIdx.x * (uint64_t)THREADS + threadIdx.x) / 32;
    if (w < p.n_row_warps)
        row_warp<T, false>(p, w);
    else if (w - p.n_row_warps < p.blk_units * 2 * p.pool.n_kv_heads)
        block_warp<T>(p, w - p.n_row_warps);
    __threadfence();
}

}  // namespace

}  // namespace tutti

using namespace tutti;

extern "C" {

// What the call refuses, from the geometry and the arguments alone.
int tutti_append_check_(const tutti_geom_t *g, const tutti_step_t *step, const tutti_tokens_t *t, const tutti_rope_t *r) {
    if (!g || !t) return TUTTI_EINVAL;
    if (int rc = check_step(step)) return rc;
    if (g->elem_bytes != 1 && g->elem_bytes != 2) return TUTTI_EINVAL;
    if (g->head_dim % 16 || g->head_dim > 256) return TUTTI_EINVAL;
    if (t->dtype != TUTTI_DTYPE_BF16 && t->dtype != TUTTI_DTYPE_FP16) return TUTTI_EINVAL;
    if (t->n_q_heads % g->n_kv_heads || t->n_q_heads > 65536) return TUTTI_EINVAL;
    if (r) {
        if (r->style != TUTTI_ROPE_HALF && r->style != TUTTI_ROPE_PAIRS) return TUTTI_EINVAL;
        if (!r->rot_dim || r->rot_dim % 16 || r->rot_dim > g->head_dim) return TUTTI_EINVAL;
        if (!r->table || ((uint64_t)r->table & 15) || !r->n_pos) return TUTTI_EINVAL;
    }
    if (!step->n_tok || !step->n_seq) return TUTTI_OK;
    if (!rows_ok(t->k, t->k_stride, g->n_kv_heads, g->head_dim) || !rows_ok(t->v, t->v_stride, g->n_kv_heads, g->head_dim))
        return TUTTI_EINVAL;
    if (t->n_q_heads) {
        if (!rows_ok(t->q, t->q_stride, t->n_q_heads, g->head_dim) ||
            !rows_ok(t->q_out, t->q_out_stride, t->n_q_heads, g->head_dim))
            return TUTTI_EINVAL;
        // in place means row by row: with another stride a row would land on one not read yet
        if (t->q == t->q_out && t->q_stride != t->q_out_stride && step->n_tok > 1) return TUTTI_EINVAL;
    } else if (t->q || t->q_out) {
        return TUTTI_EINVAL;
    }
    return TUTTI_OK;
}

// The kernels' own checks of a sequence's tables and of a block id, on host arrays.
int tutti_seq_view_(const tutti_step_t *step, uint32_t block_tokens, uint32_t s, uint32_t *out4) {
    StepDev st{step->n_seq, step->n_tok, step->n_blk, step->max_new, step->q_start, step->ctx_len,
               step->blk_start, step->block_ids, nullptr};
    SeqView v{0, 0, 0, 0};
    const int rc = seq_view(st, block_tokens, s, v);
    out4[0] = v.q0;
    out4[1] = v.n_new;
    out4[2] = v.ctx;
    out4[3] = v.b0;
    return rc;
}
int64_t tutti_block_offset_(uint32_t n_blocks, uint64_t block_stride, int32_t id) {
    PoolView p{};
    p.n_blocks = n_blocks;
    p.block_stride = block_stride;
    return block_offset(p, id);
}

int tutti_kv_append_layer(tutti_ctx_t *ctx, uint32_t layer, const tutti_step_t *step,
                          const tutti_tokens_t *t, const tutti_rope_t *r, void *stream) {
    if (!ctx) return TUTTI_EINVAL;
    if (int rc = tutti_append_check_(tutti_ctx_geom_(ctx), step, t, r)) return rc;
    AppendParams p;
    uint32_t elem_bytes;
    if (int rc = tutti_ctx_pool_view_(ctx, layer, &p.pool, &elem_bytes)) return rc;
    if (!step->n_tok || !step->n_seq) return TUTTI_OK;
    p.step = StepDev{step->n_seq, step->n_tok, step->n_blk, step->max_new, step->q_start, step->ctx_len,
                     step->blk_start, step->block_ids, step->status};
    p.rope = RopeDev{0, 0, 0, nullptr};
    if (r) p.rope = RopeDev{r->rot_dim, r->style == TUTTI_ROPE_PAIRS,
                            (uint32_t)(r->n_pos < 0x7fffffff ? r->n_pos : 0x7fffffff), r->table};
    p.n_q_heads = t->n_q_heads;
    p.q_stride = 2 * t->q_stride;
    p.k_stride = 2 * t->k_stride;
    p.v_stride = 2 * t->v_stride;
    p.q_out_stride = 2 * t->q_out_stride;
    p.q = (const char *)t->q;
    p.k = (const char *)t->k;
    p.v = (const char *)t->v;
    p.q_out = (char *)t->q_out;
    p.jobs = p.pool.head_dim / 16;
    const uint32_t per = 32 / p.jobs;
    const uint32_t rows = t->n_q_heads + (elem_bytes == 2 ? 2 * p.pool.n_kv_heads : 0);
    const uint32_t passes = (rows + per - 1) / per;
    p.row_units = (uint64_t)step->n_tok * rows > ROWS_ENOUGH ? (passes + PASSES - 1) / PASSES : passes;
    p.row_passes = p.row_units ? (passes + p.row_units - 1) / p.row_units : 0;
    uint64_t warps = (uint64_t)step->n_tok * p.row_units;
    p.blk_units = 0;
    uint64_t blk_warps = 0;
    if (elem_bytes == 1) {
        const uint64_t units = step->n_tok / p.pool.block_tokens + 2ull * step->n_seq;
        blk_warps = units * 2 * p.pool.n_kv_heads;
        p.blk_units = (uint32_t)units;
    }
    if (warps + blk_warps > 0x7fffffffull) return TUTTI_EINVAL;
    p.n_row_warps = (uint32_t)warps;
    const uint32_t grid = (uint32_t)((warps + blk_warps + THREADS / 32 - 1) / (THREADS / 32));
    OnDevice on(tutti_ctx_device_(ctx));
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    const bool bf = t->dtype == TUTTI_DTYPE_BF16;
    cudaStream_t st = (cudaStream_t)stream;
    const auto kernel = elem_bytes == 2 ? (bf ? append_kernel<__nv_bfloat16> : append_kernel<__half>)
                                        : (bf ? append8_kernel<__nv_bfloat16> : append8_kernel<__half>);
    const cudaError_t e = launch_plain(kernel, grid, THREADS, 0, st, p);
    return e == cudaSuccess ? TUTTI_OK : fail(e, "append launch");
}

}  // extern "C"
