// Copies of blocks inside the pool, in many layers at once.  Bound: HBM, every byte is read and written once.
#include "tutti_async.h"
#include "tutti_attend.h"
#include "tutti_internal.h"

namespace tutti {

namespace {

// A CTA an SM; WARPS of its warps each run a ring of STAGES stages through which bulk copies bring pieces of blocks
// in and take them out again, so few threads keep 192 KB of an SM in flight; the other warps copy scales.
constexpr int WARPS = 4, STAGES = 3, THREADS = 256;
constexpr uint32_t STAGE = 16384;
constexpr uint32_t LEAST = 2048;                // bytes that a block is cut into where there is too little to do
constexpr uint32_t LIST = 2048;                 // pairs that are taken in a round
constexpr uint32_t PER_LANE = LIST / THREADS;
constexpr uint32_t OFF_LIST = WARPS * STAGES * STAGE;
constexpr uint32_t OFF_TO = OFF_LIST + LIST * 8;                    // [warp][stage][lane] destinations,
constexpr uint32_t OFF_BYTES = OFF_TO + WARPS * STAGES * 32 * 8;    // and bytes, of the pieces in flight
constexpr uint32_t OFF_BAR = OFF_BYTES + WARPS * STAGES * 32 * 4;
constexpr uint32_t SMEM = OFF_BAR + WARPS * STAGES * 8 + THREADS / 32 * 4;

constexpr uint32_t LAYERS = 64;                 // of a launch: they travel with its parameters

struct CopyBlocks {
    LayerBytes layer[LAYERS];
    uint32_t n_layers, n_kv_heads;
    bool scales;                                // a layer has some
    uint64_t block_bytes;
    const int2 *pairs;
    const uint32_t *n_pairs;
    uint32_t max_pairs;
    int32_t *status;
};

__global__ void __launch_bounds__(THREADS, 1) copy_blocks_kernel(const __grid_constant__ CopyBlocks p) {
    extern __shared__ __align__(128) unsigned char smem[];
    int2 *list = reinterpret_cast<int2 *>(smem + OFF_LIST);
    uint32_t *counts = reinterpret_cast<uint32_t *>(smem + OFF_BAR + WARPS * STAGES * 8);
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t bars = smem_u32(smem + OFF_BAR) + warp * STAGES * 8;
    if (warp < WARPS && lane == 0) {
        for (int i = 0; i < STAGES; ++i) mbar_init(bars + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    const uint32_t n_pairs = p.n_pairs ? min(*p.n_pairs, p.max_pairs) : p.max_pairs;
    uint32_t phases = 0;                        // of the stages' barriers
    bool dead = false;
    for (uint32_t p0 = 0; p0 < n_pairs; p0 += LIST) {
        // The pairs of this round that are copied, in order: all CTAs make the same list.  A warp looks at LIST / 8 of them.
        int2 e[PER_LANE];
        uint32_t takes[PER_LANE], mine_n = 0;
#pragma unroll
        for (uint32_t k = 0; k < PER_LANE; ++k) {
            const uint32_t i = p0 + (warp * PER_LANE + k) * 32 + lane;
            e[k] = i < n_pairs ? p.pairs[i] : make_int2(-1, -1);
        }
#pragma unroll
        for (uint32_t k = 0; k < PER_LANE; ++k) {
            takes[k] = __ballot_sync(0xffffffffu, e[k].x != -1 && e[k].x != e[k].y);
            mine_n += __popc(takes[k]);
        }
        if (lane == 0) counts[warp] = mine_n;
        __syncthreads();
        uint32_t n = 0, at = 0;
#pragma unroll
        for (uint32_t w = 0; w < THREADS / 32; ++w) {
            if (w == warp) at = n;
            n += counts[w];
        }
#pragma unroll
        for (uint32_t k = 0; k < PER_LANE; ++k) {
            if (takes[k] >> lane & 1) list[at + __popc(takes[k] & ((1u << lane) - 1))] = e[k];
            at += __popc(takes[k]);
        }
        __syncthreads();
        if (warp >= WARPS) {
            // scales: float by float, few
            const uint64_t per_layer = (uint64_t)n * 2 * p.n_kv_heads, total = p.scales ? per_layer * p.n_layers : 0;
            for (uint64_t i = (uint64_t)blockIdx.x * (THREADS - 32 * WARPS) + threadIdx.x - 32 * WARPS; i < total; i += (uint64_t)gridDim.x * (THREADS - 32 * WARPS)) {
                const uint32_t layer = (uint32_t)(i / per_layer), j = (uint32_t)(i % per_layer);
                const uint32_t h = j % p.n_kv_heads, half = j / p.n_kv_heads % 2;
                const int2 e = list[j / p.n_kv_heads / 2];
                const LayerBytes &l = p.layer[layer];
                float *s = half ? l.v_scale : l.k_scale;
                if (s && (uint32_t)e.x < l.n_blocks && (uint32_t)e.y < l.n_blocks)
                    s[(uint64_t)(uint32_t)e.y * l.scale_row + h] = s[(uint64_t)(uint32_t)e.x * l.scale_row + h];
            }
        } else if (!dead) {
            const uint64_t halves = (uint64_t)n * 2 * p.n_layers;
            const uint32_t agents = gridDim.x * WARPS, agent = warp * gridDim.x + blockIdx.x;
            // pieces of `piece` bytes, the last of a block the rest
            uint32_t piece = (uint32_t)min(p.block_bytes, (uint64_t)STAGE);
            while (piece > LEAST && halves * ((p.block_bytes + piece - 1) / piece) < agents) piece = (piece / 2 + 15) & ~15u;
            const uint32_t parts = (uint32_t)((p.block_bytes + piece - 1) / piece);
            const uint64_t pieces = halves * parts;
            const uint32_t fit = min(32u, STAGE / piece);
            const uint32_t per = (uint32_t)min((uint64_t)fit, (pieces + agents - 1) / agents);     // pieces a stage
            const uint64_t units = per ? (pieces + per - 1) / per : 0;
            unsigned long long *to = reinterpret_cast<unsigned long long *>(smem + OFF_TO) + warp * STAGES * 32 + lane;
            uint32_t *bytes = reinterpret_cast<uint32_t *>(smem + OFF_BYTES) + warp * STAGES * 32 + lane;
            const uint32_t ring = smem_u32(smem) + warp * STAGES * STAGE;
            auto issue = [&](uint64_t unit, uint32_t stage) {
                const uint64_t i = unit * per + lane;
                uint32_t size = 0;
                unsigned long long src = 0;
                if (unit < units && lane < per && i < pieces) {
                    const uint32_t part = (uint32_t)(i % parts);
                    const uint64_t h = i / parts, half = h % 2, pair = h / 2 % n;
                    const LayerBytes &pool = p.layer[h / 2 / n];
                    const int2 e = list[pair];
                    if ((uint32_t)e.x < pool.n_blocks && (uint32_t)e.y < pool.n_blocks) {
                        const uint64_t base = (half ? pool.v_base : pool.k_base) + (uint64_t)part * piece;
                        size = (uint32_t)min((uint64_t)piece, p.block_bytes - (uint64_t)part * piece);
                        src = base + (uint32_t)e.x * pool.block_stride;
                        to[stage * 32] = base + (uint32_t)e.y * pool.block_stride;
                    } else {
                        if (p.status) atomicCAS(p.status, TUTTI_OK, TUTTI_EFAULT);
                    }
                }
                bytes[stage * 32] = size;
                const uint32_t all = __reduce_add_sync(0xffffffffu, size);
                if (lane == 0) mbar_expect_tx(bars + 8 * stage, all);
                __syncwarp();
                if (size) bulk_g2s(ring + stage * STAGE + lane * piece, src, size, bars + 8 * stage);
            };
            const uint64_t mine = units > agent ? (units - agent + agents - 1) / agents : 0;
            for (uint32_t k = 0; k < STAGES - 1; ++k)
                if (k < mine) issue(agent + (uint64_t)k * agents, k);
            uint32_t stage = 0;
            for (uint64_t k = 0; k < mine; ++k) {
                const uint32_t bar = bars + 8 * stage;
                bool there = mbar_wait_bounded(bar, phases >> stage & 1);
                if (!__all_sync(0xffffffffu, there)) {
                    if (p.status) atomicCAS(p.status, TUTTI_OK, TUTTI_ETIMEDOUT);
                    for (int s = 0; s < STAGES; ++s) (void)mbar_wait_bounded(bars + 8 * s, phases >> s & 1);      // copies in flight
                    dead = true;
                    break;
                }
                phases ^= 1u << stage;
                if (const uint32_t size = bytes[stage * 32]) bulk_s2g(to[stage * 32], ring + stage * STAGE + lane * piece, size);
                bulk_commit();
                const uint32_t next = stage == 0 ? STAGES - 1 : stage - 1;
                if (k + STAGES - 1 < mine) {
                    bulk_wait_read_1();         // the stage before this one has been read
                    __syncwarp();
                    issue(agent + (k + STAGES - 1) * agents, next);
                }
                stage = stage + 1 == STAGES ? 0 : stage + 1;
            }
            bulk_wait_all();
        }
        __syncthreads();
    }
}

}  // namespace

cudaError_t copy_blocks_setup() {
    return cudaFuncSetAttribute(copy_blocks_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
}

}  // namespace tutti

using namespace tutti;

extern "C" {

// What the call refuses, from the arguments alone.
int tutti_copy_check_(const tutti_geom_t *g, uint32_t first_layer, uint32_t n_layers, const int32_t *pairs, uint32_t max_pairs, const uint32_t *n_pairs,
                      const int32_t *status) {
    if (!g || first_layer > g->n_layers || n_layers > g->n_layers - first_layer || max_pairs > 0x7fffffffu) return TUTTI_EINVAL;
    if (max_pairs && (!pairs || ((uint64_t)pairs & 7))) return TUTTI_EINVAL;
    return ((uint64_t)n_pairs | (uint64_t)status) & 3 ? TUTTI_EINVAL : TUTTI_OK;
}

int tutti_kv_copy_blocks(tutti_ctx_t *ctx, uint32_t first_layer, uint32_t n_layers, const int32_t *pairs, uint32_t max_pairs, const uint32_t *n_pairs,
                         int32_t *status, void *stream) {
    if (!ctx) return TUTTI_EINVAL;
    const tutti_geom_t *g = tutti_ctx_geom_(ctx);
    if (int rc = tutti_copy_check_(g, first_layer, n_layers, pairs, max_pairs, n_pairs, status)) return rc;
    CopyBlocks p;
    for (uint32_t l = 0; l < n_layers; ++l)
        if (!tutti_ctx_layer_bytes_(ctx, first_layer + l, &p.layer[l % LAYERS])) return TUTTI_EINVAL;
    if (!n_layers || !max_pairs) return TUTTI_OK;
    p.n_kv_heads = g->n_kv_heads;
    p.block_bytes = (uint64_t)g->block_tokens * g->n_kv_heads * g->head_dim * g->elem_bytes;
    p.pairs = reinterpret_cast<const int2 *>(pairs);
    p.n_pairs = n_pairs;
    p.max_pairs = max_pairs;
    p.status = status;
    OnDevice on(tutti_ctx_device_(ctx));
    if (!on.ok) return fail(cudaErrorInvalidDevice, "cudaSetDevice");
    for (uint32_t l0 = 0; l0 < n_layers; l0 += LAYERS) {
        p.n_layers = n_layers - l0 < LAYERS ? n_layers - l0 : LAYERS;
        p.scales = false;
        for (uint32_t l = 0; l < p.n_layers; ++l) {
            tutti_ctx_layer_bytes_(ctx, first_layer + l0 + l, &p.layer[l]);
            p.scales = p.scales || p.layer[l].k_scale;
        }
        const cudaError_t e = launch_plain(copy_blocks_kernel, tutti_ctx_sms_(ctx), THREADS, SMEM, (cudaStream_t)stream, p);
        if (e != cudaSuccess) return fail(e, "copy launch");
    }
    return TUTTI_OK;
}

}  // extern "C"
