// Shared by the attention kernels: the call's parameters and a few instructions.
#pragma once
#include <cuda_fp8.h>

#include "tutti_paged.h"

namespace tutti {

struct AttendParams {
    StepDev step;
    PoolView pool;
    uint32_t n_q_heads, group;
    uint64_t q_stride, out_stride;    // elements
    const void *q;
    void *out;
    float *lse;
    float scale;
    uint32_t group_mul, group_shift;  // row / group = row * group_mul >> group_shift
    uint32_t window, sinks;           // window 0: every key up to the row's own
    // Many rows: a tile's keys are the first `front` of the sequence (the sinks, up to a multiple of `grain`) and the ones
    // from its window on, which begins at a multiple of it; a tensor copy brings `grain` rows of one block or a multiple.
    uint32_t front, grain;

    // The first key behind the first `sinks` that a row at position `first` (any row behind it) sees: 0 or less, all.
    __host__ __device__ int64_t window_start(int64_t first) const { return first - window + 1; }

    __host__ __device__ uint32_t token_of(uint32_t row) const { return (uint32_t)((uint64_t)row * group_mul >> group_shift); }
    __host__ __device__ uint32_t member_of(uint32_t row) const { return row - token_of(row) * group; }
};

__host__ __device__ inline uint32_t grain_of(uint32_t block_tokens) { return 64 % block_tokens == 0 ? block_tokens : block_tokens % 64 == 0 ? 64 : 16; }
__host__ __device__ inline uint32_t front_of(uint32_t sinks, uint32_t grain) { return (sinks + grain - 1) / grain * grain; }

// Tile loads of the layer's keys and values.
struct PoolMaps {
    CUtensorMap k, v;
    bool valid;
};

// Where parts of a tile that several workers share are left for the last of them to join.
struct Workspace {
    float *part;            // two slots a worker: rows x D sums, then behind them all maximum and denominator
    uint32_t *count;        // parts that have arrived at the tile that starts in a worker; zero between calls
    uint32_t workers;
};

// a / b, by the much faster 32-bit division where both fit (they nearly always do)
__host__ __device__ inline unsigned long long quotient(unsigned long long a, unsigned long long b) {
    return (a | b) >> 32 ? a / b : (uint32_t)a / (uint32_t)b;
}

#ifdef __CUDACC__
// One arrival: what this thread has seen of its CTA (behind a barrier) is released with it, and what the
// earlier arrivals released is acquired.
__device__ inline uint32_t arrive_gpu(uint32_t *count) {
    uint32_t old;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(old) : "l"(count) : "memory");
    return old;
}
__device__ inline float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ inline uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ inline void cp16(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ inline void cp4(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ inline void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ inline void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// four e4m3 codes as four f16
__device__ inline void codes4(uint32_t w, uint32_t &lo, uint32_t &hi) {
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
}
#endif

// 8 or 16 rows a tile (tutti_attend_few.cu).
constexpr int FEW_ROWS = 16;
cudaError_t few_setup();
cudaError_t few_launch(const AttendParams &p, const Workspace &ws, int sms, bool c8, bool bf, cudaStream_t st);
size_t few_part_bytes(int sms);
uint32_t few_workers(int sms);

// 256 rows a tile (tutti_attend_many.cu).
cudaError_t many_setup();
cudaError_t many_launch(const AttendParams &p, const PoolMaps &maps, const Workspace &ws, bool c8, bool bf, cudaStream_t st);
size_t many_part_bytes(uint32_t workers);
uint32_t many_workers(int sms);

}  // namespace tutti
