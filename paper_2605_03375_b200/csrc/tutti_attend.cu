// Entry points of attention over the paged pool:
//     out = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q . k_j - m),   m = max_j scale q . k_j
// over the keys j <= position of the row.
#include <cmath>
#include <new>

#include "tutti_attend.h"

using namespace tutti;

struct tutti_attn {
    tutti_ctx *ctx;
    int device;
    Workspace few, many;     // they share the parts' memory
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
    if ((uint64_t)step->n_tok * io->n_q_heads > 0x7fffffffull) return TUTTI_EINVAL;
    if (!step->n_tok || !step->n_seq) return TUTTI_OK;
    if (io->q == io->out) return TUTTI_EINVAL;
    if (!rows_ok(io->q, io->q_stride, io->n_q_heads, g->head_dim) ||
        !rows_ok(io->out, io->out_stride, io->n_q_heads, g->head_dim) || ((uint64_t)io->lse & 3))
        return TUTTI_EINVAL;
    return TUTTI_OK;
}

int tutti_attn_create(tutti_ctx_t *ctx, tutti_attn_t **out) {
    if (!ctx || !out) return TUTTI_EINVAL;
    OnDevice on(tutti_ctx_device_(ctx));
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    cudaError_t e = few_setup();
    if (e == cudaSuccess) e = many_setup();
    if (e != cudaSuccess) return fail(e, "cudaFuncSetAttribute");
    tutti_attn *a = new (std::nothrow) tutti_attn();
    if (!a) return TUTTI_ENOMEM;
    a->ctx = ctx;
    a->device = tutti_ctx_device_(ctx);
    const uint32_t n_few = few_workers(tutti_ctx_sms_(ctx)), n_many = many_workers(tutti_ctx_sms_(ctx));
    const size_t few_part = few_part_bytes(tutti_ctx_sms_(ctx)), many_part = many_part_bytes(n_many), part = few_part > many_part ? few_part : many_part;
    const size_t counts = (n_few + 2 * n_many) * sizeof(uint32_t);
    float *parts = nullptr;
    uint32_t *count = nullptr;
    if ((e = cudaMalloc((void **)&parts, part)) != cudaSuccess || (e = cudaMalloc((void **)&count, counts)) != cudaSuccess ||
        (e = cudaMemset(count, 0, counts)) != cudaSuccess || (e = cudaDeviceSynchronize()) != cudaSuccess) {
        if (parts) cudaFree(parts);
        if (count) cudaFree(count);
        delete a;
        fail(e, "attention workspace");
        return TUTTI_ENOMEM;
    }
    a->few = Workspace{parts, count, n_few};
    a->many = Workspace{parts, count + n_few, n_many};
    *out = a;
    return TUTTI_OK;
}

int tutti_attn_destroy(tutti_attn_t *a) {
    if (!a) return TUTTI_EINVAL;
    OnDevice on(a->device);
    cudaDeviceSynchronize();
    cudaFree(a->few.part);
    cudaFree(a->few.count);
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
    division_by(p.group, p.group_mul, p.group_shift);
    p.q_stride = io->q_stride;
    p.out_stride = io->out_stride;
    p.q = io->q;
    p.out = io->out;
    p.lse = io->lse;
    p.scale = io->scale;
    OnDevice on(tutti_ctx_device_(a->ctx));
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    const bool bf = io->dtype == TUTTI_DTYPE_BF16;
    const bool few = (uint64_t)step->max_new * p.group <= FEW_ROWS;
    PoolMaps maps;
    if (!few) maps.valid = tutti_ctx_pool_maps_(a->ctx, layer, &maps.k, &maps.v);
    const cudaError_t e = few ? few_launch(p, a->few, tutti_ctx_sms_(a->ctx), elem_bytes == 1, bf, (cudaStream_t)stream)
                              : many_launch(p, maps, a->many, elem_bytes == 1, bf, (cudaStream_t)stream);
    return e == cudaSuccess ? TUTTI_OK : fail(e, "attend launch");
}

}  // extern "C"
