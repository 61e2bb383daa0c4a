// What the operators that compute on the paged pool (append, attend) share: the device view of
// a registered pool layer and of a step's tables, and the checks that keep every access inside
// them.  The checks are plain arithmetic, callable on the host too.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <string>

#include "../../include/tutti.h"

namespace tutti {

struct PoolView {
    uint64_t k_base, v_base, block_stride;
    uint32_t n_blocks, block_tokens, n_kv_heads, head_dim;
    uint64_t tok_stride, head_stride;       // bytes between tokens / heads of a block
    float *k_scale, *v_scale;               // [n_blocks][scale_row], 8-bit pools only
    bool hnd;                               // head-major blocks
    uint32_t scale_row;                     // n_kv_heads or more
    uint32_t block_mul, block_shift;        // key / block_tokens = key * block_mul >> block_shift, for keys below 2^31

    __host__ __device__ uint32_t block_of(uint32_t key) const { return (uint32_t)((uint64_t)key * block_mul >> block_shift); }
    __host__ __device__ uint32_t row_of(uint32_t key) const { return key - block_of(key) * block_tokens; }
};

// n / d for n < 2^31 as a product and a shift (Granlund and Montgomery): with 2^s >= d the
// multiplier floor(2^(31+s) / d) + 1 fits 32 bits and errs by less than 2^s / 2^31 a unit of n.
inline void division_by(uint32_t d, uint32_t &mul, uint32_t &shift) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    shift = 31 + s;
    mul = (uint32_t)((1ull << shift) / d + (d > 1 ? 1 : 0));
}

// Tensor maps of a pool layer, by pool layout (TUTTI_POOL_NHD, TUTTI_POOL_HND).
struct PoolTensorMaps {
    CUtensorMap k[2], v[2];
    bool valid[2] = {false, false};
};

struct StepDev {
    uint32_t n_seq, n_tok, n_blk, max_new;
    const uint32_t *q_start, *ctx_len, *blk_start;
    const int32_t *block_ids;
    int32_t *status;
};

struct SeqView {
    uint32_t q0, n_new;     // first row and number of rows of the step's token arrays
    uint32_t ctx;           // tokens in the cache, the new ones included
    uint32_t b0;            // first entry of block_ids
};

// The tables of one sequence; anything but TUTTI_OK means that its numbers contradict each
// other or the step's sizes, and nothing may be read or written for it.
__host__ __device__ inline int seq_view(const StepDev &st, uint32_t block_tokens, uint32_t s, SeqView &v) {
    const uint32_t q0 = st.q_start[s], q1 = st.q_start[s + 1];
    const uint32_t b0 = st.blk_start[s], b1 = st.blk_start[s + 1];
    const uint32_t ctx = st.ctx_len[s];
    if (q0 > q1 || q1 > st.n_tok || q1 - q0 > st.max_new) return TUTTI_EINVAL;
    if (b0 > b1 || b1 > st.n_blk || ctx > 0x7fffffffu) return TUTTI_EINVAL;
    if ((ctx + block_tokens - 1) / block_tokens > b1 - b0) return TUTTI_EINVAL;
    v.q0 = q0;
    v.n_new = q1 - q0;
    v.ctx = ctx;
    v.b0 = b0;
    return TUTTI_OK;
}

// Byte offset of block `id` from a layer's base, or -1 for an id outside the pool.
__host__ __device__ inline int64_t block_offset(const PoolView &p, int32_t id) {
    return (uint32_t)id < p.n_blocks ? (int64_t)((uint64_t)(uint32_t)id * p.block_stride) : -1;
}

#ifdef __CUDACC__
// two 32-bit numbers, each rounded once
__device__ inline uint32_t pack2(float a, float b, __nv_bfloat16) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&h);
}
__device__ inline uint32_t pack2(float a, float b, __half) {
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&h);
}

__device__ inline void report(const StepDev &st, int code) {
    if (st.status) atomicCAS(st.status, TUTTI_OK, code);
}

// Largest s with start(s) <= x over s in [0, n): all lanes of a warp, 128 probes a round (one round of
// loads for up to 128 sequences).  start(0) <= x is taken for granted; the caller checks what it found.
template <typename F>
__device__ inline uint32_t warp_find(uint32_t n, uint32_t x, F start) {
    const uint32_t lane = threadIdx.x & 31;
    uint32_t lo = 0, len = n;
    while (len > 1) {
        const uint32_t step = (len + 127) / 128;
        bool le[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t at = (lane * 4 + k) * step;
            le[k] = at < len && start(lo + at) <= x;
        }
        uint32_t n_le = 0;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) n_le += __popc(__ballot_sync(0xffffffffu, le[k]));
        const uint32_t last = n_le ? n_le - 1 : 0;
        lo += last * step;
        len = len - last * step < step ? len - last * step : step;
    }
    return lo;
}
#endif

}  // namespace tutti

// The layer's view and the context's device, for the operators' entry points (tutti_lib.cu).
struct tutti_ctx;
extern "C" int tutti_ctx_pool_view_(tutti_ctx *ctx, uint32_t layer, tutti::PoolView *view, uint32_t *elem_bytes);
extern "C" bool tutti_ctx_pool_maps_(tutti_ctx *ctx, uint32_t layer, CUtensorMap *k, CUtensorMap *v);
extern "C" int tutti_ctx_device_(tutti_ctx *ctx);
extern "C" int tutti_ctx_sms_(tutti_ctx *ctx);
extern "C" const tutti_geom_t *tutti_ctx_geom_(tutti_ctx *ctx);
extern "C" void tutti_set_cuda_error_(const char *msg);

namespace tutti {

// Argument checks that need no device (the entry points call them first).
inline int check_step(const tutti_step_t *st) {
    if (!st) return TUTTI_EINVAL;
    if (st->n_tok > 0x7fffffffu || st->n_seq > 0x3fffffffu || st->n_blk > 0x7fffffffu) return TUTTI_EINVAL;
    if (st->n_seq && (!st->q_start || !st->ctx_len || !st->blk_start)) return TUTTI_EINVAL;
    if (st->n_blk && !st->block_ids) return TUTTI_EINVAL;
    if (st->n_tok && st->n_seq && !st->max_new) return TUTTI_EINVAL;
    if (((uint64_t)st->q_start | (uint64_t)st->ctx_len | (uint64_t)st->blk_start |
         (uint64_t)st->block_ids | (uint64_t)st->status) & 3)
        return TUTTI_EINVAL;
    return TUTTI_OK;
}

// [n_tok][heads][head_dim] 16-bit elements at p, `stride` elements from token to token.
inline bool rows_ok(const void *p, uint64_t stride, uint64_t heads, uint64_t head_dim) {
    return p && ((uint64_t)p & 15) == 0 && stride % 8 == 0 && stride >= heads * head_dim && stride < (1ull << 31);
}

inline int fail(cudaError_t e, const char *what) {
    tutti_set_cuda_error_((std::string(what) + ": " + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")").c_str());
    return TUTTI_ECUDA;
}

// A launch whose own status is returned: an error that another call of the program left behind is
// neither taken for this launch's nor cleared.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_plain(void (*kernel)(KArgs...), uint32_t grid, uint32_t block, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Makes a device current for a scope.
struct OnDevice {
    int prev = -1, target;
    bool ok;
    explicit OnDevice(int dev) : target(dev) {
        ok = cudaGetDevice(&prev) == cudaSuccess && (prev == dev || cudaSetDevice(dev) == cudaSuccess);
    }
    ~OnDevice() {
        if (ok && prev != target) cudaSetDevice(prev);
    }
};

}  // namespace tutti
