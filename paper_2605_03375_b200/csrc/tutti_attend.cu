// Causal attention of a step's queries over a layer of the paged pool:
//     out = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q . k_j - m),   m = max_j scale q . k_j
// over the keys j <= position of the row.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cmath>
#include <new>
#include <string>

#include "tutti_paged.h"

namespace tutti {

namespace {

struct AttendParams {
    StepDev step;
    PoolView pool;
    uint32_t n_q_heads, group;
    uint64_t q_stride, out_stride;    // elements
    const void *q;
    void *out;
    float *lse;
    float scale;
};

template <typename T> __device__ inline float to_f(T x);
template <> __device__ inline float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ inline float to_f(__half x) { return __half2float(x); }
template <> __device__ inline float to_f(__nv_fp8_e4m3 x) { return (float)x; }
__device__ inline void from_f(float x, __nv_bfloat16 &y) { y = __float2bfloat16(x); }
__device__ inline void from_f(float x, __half &y) { y = __float2half(x); }

// One warp a row (token, query head), its lanes over the head's dimensions, one key at a time.
template <typename T, typename C>
__global__ void __launch_bounds__(256) attend_rows_kernel(const __grid_constant__ AttendParams p) {
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t w = (blockIdx.x * 256ull + threadIdx.x) / 32;
    const uint32_t tok = (uint32_t)(w / p.n_q_heads), h = (uint32_t)(w % p.n_q_heads), kh = h / p.group;
    if (tok >= p.step.n_tok || tok >= __ldg(p.step.q_start + p.step.n_seq)) return;
    const uint32_t s = warp_find(p.step.n_seq, tok, [&](uint32_t i) { return __ldg(p.step.q_start + i); });
    SeqView v;
    int code = seq_view(p.step, p.pool.block_tokens, s, v);
    if (code == TUTTI_OK && (tok < v.q0 || tok - v.q0 >= v.n_new)) code = TUTTI_EINVAL;
    if (code != TUTTI_OK) {
        if (lane == 0) report(p.step, code);
        return;
    }
    const uint32_t D = p.pool.head_dim, n = D / 32;
    float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0;
    for (uint32_t i = 0; i < n; ++i)
        q[i] = to_f(((const T *)p.q)[tok * p.q_stride + h * D + i * 32 + lane]);
    const int64_t n_keys = (int64_t)v.ctx - v.n_new + (tok - v.q0) + 1;
    for (int64_t j = 0; j < n_keys; ++j) {
        const int32_t id = __ldg(p.step.block_ids + v.b0 + j / p.pool.block_tokens);
        int64_t at = block_offset(p.pool, id);
        if (at < 0) {
            if (lane == 0) report(p.step, TUTTI_EFAULT);
            continue;
        }
        at += j % p.pool.block_tokens * p.pool.tok_stride + kh * p.pool.head_stride;
        const C *k = (const C *)(p.pool.k_base + at), *vv = (const C *)(p.pool.v_base + at);
        const float ks = sizeof(C) == 1 ? p.pool.k_scale[(uint64_t)id * p.pool.n_kv_heads + kh] : 1.0f;
        const float vs = sizeof(C) == 1 ? p.pool.v_scale[(uint64_t)id * p.pool.n_kv_heads + kh] : 1.0f;
        float x = 0;
        for (uint32_t i = 0; i < n; ++i) x += q[i] * to_f(k[i * 32 + lane]);
        for (int b = 16; b; b >>= 1) x += __shfl_xor_sync(0xffffffffu, x, b);
        x *= ks * p.scale;
        const float m2 = fmaxf(m, x), a = expf(m - m2), e = expf(x - m2);
        l = l * a + e;
        for (uint32_t i = 0; i < n; ++i) o[i] = o[i] * a + e * vs * to_f(vv[i * 32 + lane]);
        m = m2;
    }
    for (uint32_t i = 0; i < n; ++i)
        from_f(l > 0 ? o[i] / l : 0.0f, ((T *)p.out)[tok * p.out_stride + h * D + i * 32 + lane]);
    if (p.lse && lane == 0) p.lse[(uint64_t)tok * p.n_q_heads + h] = m + logf(l);
}

int fail(cudaError_t e, const char *what) {
    tutti_set_cuda_error_((std::string(what) + ": " + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")").c_str());
    return TUTTI_ECUDA;
}

}  // namespace

}  // namespace tutti

using namespace tutti;

struct tutti_attn {
    tutti_ctx *ctx;
};

extern "C" {

// What the call refuses, from the geometry and the arguments alone.
int tutti_attend_check_(const tutti_geom_t *g, const tutti_step_t *step, const tutti_attend_t *io) {
    if (!g || !io) return TUTTI_EINVAL;
    if (int rc = check_step(step)) return rc;
    if (g->elem_bytes != 1 && g->elem_bytes != 2) return TUTTI_EINVAL;
    if (g->head_dim != 64 && g->head_dim != 128) return TUTTI_EINVAL;
    if (io->dtype != TUTTI_DTYPE_BF16 && io->dtype != TUTTI_DTYPE_FP16) return TUTTI_EINVAL;
    if (!io->n_q_heads || io->n_q_heads % g->n_kv_heads || io->n_q_heads > 65536) return TUTTI_EINVAL;
    if (!std::isfinite(io->scale) || io->reserved) return TUTTI_EINVAL;
    if (!step->n_tok || !step->n_seq) return TUTTI_OK;
    if (!rows_ok(io->q, io->q_stride, io->n_q_heads, g->head_dim) ||
        !rows_ok(io->out, io->out_stride, io->n_q_heads, g->head_dim) || ((uint64_t)io->lse & 3))
        return TUTTI_EINVAL;
    return TUTTI_OK;
}

int tutti_attn_create(tutti_ctx_t *ctx, tutti_attn_t **out) {
    if (!ctx || !out) return TUTTI_EINVAL;
    tutti_attn *a = new (std::nothrow) tutti_attn();
    if (!a) return TUTTI_ENOMEM;
    a->ctx = ctx;
    *out = a;
    return TUTTI_OK;
}

int tutti_attn_destroy(tutti_attn_t *a) {
    if (!a) return TUTTI_EINVAL;
    delete a;
    return TUTTI_OK;
}

int tutti_kv_attend_layer(tutti_attn_t *a, uint32_t layer, const tutti_step_t *step,
                          const tutti_attend_t *io, void *stream) {
    if (!a) return TUTTI_EINVAL;
    if (int rc = tutti_attend_check_(tutti_ctx_geom_(a->ctx), step, io)) return rc;
    AttendParams p;
    uint32_t elem_bytes;
    if (int rc = tutti_ctx_pool_view_(a->ctx, layer, &p.pool, &elem_bytes)) return rc;
    if (!step->n_tok || !step->n_seq) return TUTTI_OK;
    p.step = StepDev{step->n_seq, step->n_tok, step->n_blk, step->max_new, step->q_start, step->ctx_len,
                     step->blk_start, step->block_ids, step->status};
    p.n_q_heads = io->n_q_heads;
    p.group = io->n_q_heads / p.pool.n_kv_heads;
    p.q_stride = io->q_stride;
    p.out_stride = io->out_stride;
    p.q = io->q;
    p.out = io->out;
    p.lse = io->lse;
    p.scale = io->scale;
    const uint64_t grid = ((uint64_t)step->n_tok * io->n_q_heads + 7) / 8;
    if (grid > 0x7fffffffull) return TUTTI_EINVAL;
    OnDevice on(tutti_ctx_device_(a->ctx));
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    cudaStream_t st = (cudaStream_t)stream;
    const bool bf = io->dtype == TUTTI_DTYPE_BF16;
    if (elem_bytes == 2) {
        if (bf) attend_rows_kernel<__nv_bfloat16, __nv_bfloat16><<<(uint32_t)grid, 256, 0, st>>>(p);
        else attend_rows_kernel<__half, __half><<<(uint32_t)grid, 256, 0, st>>>(p);
    } else {
        if (bf) attend_rows_kernel<__nv_bfloat16, __nv_fp8_e4m3><<<(uint32_t)grid, 256, 0, st>>>(p);
        else attend_rows_kernel<__half, __nv_fp8_e4m3><<<(uint32_t)grid, 256, 0, st>>>(p);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TUTTI_OK : fail(e, "attend launch");
}

}  // extern "C"
