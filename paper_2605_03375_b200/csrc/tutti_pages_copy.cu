// Copies of blocks inside the pool, in many layers at once.  Bound: HBM, every byte is read and written once.
#include "tutti_async.h"
#include "tutti_attend.h"
#include "tutti_internal.h"

namespace tutti {

namespace {

// A CTA an SM; AGENTS of its warps each run a ring of STAGES stages through which bulk copies bring pieces of blocks
// in and take them out again, so few threads keep 192 KB of an SM in flight; the next warp copies scales.
//
// Work is dealt out in tickets.  Even shares leave the fastest SMs waiting: under load the slowest moves about half as much as
// the average (2048 blocks of 32 KB in 8 layers, 2.1 GB read and written: 351 us with even shares, 331 so = 6.5 TB/s).  So a CTA
// takes tickets as it goes on, each the index of a CTA of the grid that has not been launched yet (clusterlaunchcontrol, which
// needs no counter in memory that two calls could share).  The first `width` tickets have two fifths of the work, the next two
// fifths of the rest, and so on: few tickets, the last ones small.  A call with a few us of work has no second ticket.  The grid is what
// max_pairs may need: where none of the pairs counts, a call takes 12 us for 2048 of them, 53 for 65536, 410 for 524288.
constexpr uint32_t AGENTS = 2, STAGES = 3, THREADS = 256;
constexpr uint32_t STAGE = 32768;
constexpr uint32_t LEAST = 2048;                // bytes that a block is cut into where there is too little to do
constexpr uint32_t LIST = 2048;                 // pairs that are taken in a round
constexpr uint32_t PER_LANE = LIST / THREADS;
constexpr uint32_t SLOTS = 4;                   // tickets between the first and the last warp
constexpr uint32_t MOST_LEVELS = 10, LAST_TICKET = 65536;            // bytes that the smallest tickets have at least
constexpr uint32_t OFF_LIST = AGENTS * STAGES * STAGE;
constexpr uint32_t OFF_TO = OFF_LIST + LIST * 8;                    // [agent][stage][lane] destinations,
constexpr uint32_t OFF_BYTES = OFF_TO + AGENTS * STAGES * 32 * 8;   // and bytes, of the pieces in flight
constexpr uint32_t OFF_SLOT = OFF_BYTES + AGENTS * STAGES * 32 * 4; // [SLOTS] answers to requests for a ticket
constexpr uint32_t OFF_BAR = OFF_SLOT + SLOTS * 16;                 // [agent][stage] loads, [SLOTS] answers, [SLOTS] their readers
constexpr uint32_t OFF_COUNT = OFF_BAR + (AGENTS * STAGES + 2 * SLOTS) * 8;
constexpr uint32_t OFF_CLAIM = OFF_COUNT + THREADS / 32 * 4;        // [2 SLOTS] units of a ticket that an agent has taken
constexpr uint32_t SMEM = OFF_CLAIM + 2 * SLOTS * 4;
constexpr uint32_t LAYERS = 64;                 // of a launch: they travel with its parameters

struct CopyBlocks {
    LayerBytes layer[LAYERS];
    uint32_t n_layers, n_kv_heads;
    bool scales;                                // a layer has some
    uint64_t block_bytes;
    const int2 *pairs;
    const uint32_t *n_pairs;
    uint32_t max_pairs;
    uint32_t width, levels;                     // tickets of a level, levels of a round
    int32_t *status;
};

// The units at, at + width, ... below `end` of `units` that ticket `t` of a round has.
__host__ __device__ inline void ticket_units(uint64_t units, uint32_t t, uint32_t width, uint32_t levels, uint64_t &at, uint64_t &end) {
    uint64_t left = units;                      // behind the levels in front
    for (uint32_t l = t / width; l; --l) left = left * 3 / 5;
    at = units - left + t % width;
    end = t / width + 1 == levels ? units : units - left * 3 / 5;
}

// Asks for a CTA that has not been launched; the answer (16 bytes) completes on `bar`.
__device__ inline void ask(uint32_t slot, uint32_t bar) {
    mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(slot), "r"(bar) : "memory");
}
// Whether there was one, and its index.
__device__ inline bool answer(uint32_t slot, uint32_t &index) {
    uint32_t ok, x;
    asm volatile("{\n.reg .b128 a;\n.reg .pred p;\nld.shared.b128 a, [%2];\n"
                 "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\nselp.u32 %0, 1, 0, p;\nmov.u32 %1, 0;\n"
                 "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, _, _, _}, a;\n}"
                 : "=r"(ok), "=r"(x) : "r"(slot) : "memory");
    index = x;
    return ok;
}

__global__ void __launch_bounds__(THREADS, 1) copy_blocks_kernel(const __grid_constant__ CopyBlocks p) {
    extern __shared__ __align__(128) unsigned char smem[];
    int2 *list = reinterpret_cast<int2 *>(smem + OFF_LIST);
    uint32_t *counts = reinterpret_cast<uint32_t *>(smem + OFF_COUNT);
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t base = smem_u32(smem), bars = base + OFF_BAR + warp * STAGES * 8;       // of an agent
    const uint32_t full = base + OFF_BAR + AGENTS * STAGES * 8, empty = full + SLOTS * 8;
    uint32_t *claims = reinterpret_cast<uint32_t *>(smem + OFF_CLAIM);
    if (threadIdx.x < 2 * SLOTS) claims[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < AGENTS * STAGES + SLOTS; ++i) mbar_init(base + OFF_BAR + 8 * i, 1);
        for (uint32_t i = 0; i < SLOTS; ++i) mbar_init(empty + 8 * i, THREADS / 32);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t n_pairs = p.n_pairs ? min(*p.n_pairs, p.max_pairs) : p.max_pairs;
    const uint32_t a_round = p.width * p.levels;

    // ---- this warp's walk over the CTA's tickets, and over its units of each ----
    uint32_t ticket = blockIdx.x, n_tickets = 0, round = ~0u, n = 0;
    bool open = true;
    bool asks = gridDim.x > p.width;            // or the CTAs of the grid are the only tickets
    if (threadIdx.x == 0 && asks) ask(base + OFF_SLOT, full);
    // Pieces of `piece` bytes (the last of a block the rest), `per` of them a unit; the ticket's units.
    uint32_t piece = 0, parts = 0, per = 0;
    uint64_t pieces = 0, at = 0, end = 0;
    auto give_up = [&]() {
        if (p.status) atomicCAS(p.status, TUTTI_OK, TUTTI_ETIMEDOUT);
        open = false;
    };
    // The pairs of a round that are copied, in order: all CTAs make the same list.  All warps of the CTA come here together.
    auto list_pairs = [&](uint32_t p0) {
        int2 e[PER_LANE];
        uint32_t takes[PER_LANE], mine = 0;
#pragma unroll
        for (uint32_t k = 0; k < PER_LANE; ++k) {
            const uint32_t i = p0 + (warp * PER_LANE + k) * 32 + lane;
            e[k] = i < n_pairs ? p.pairs[i] : make_int2(-1, -1);
        }
        __syncthreads();                        // the list of the round before is not needed any longer
#pragma unroll
        for (uint32_t k = 0; k < PER_LANE; ++k) {
            takes[k] = __ballot_sync(0xffffffffu, e[k].x != -1 && e[k].x != e[k].y);
            mine += __popc(takes[k]);
        }
        if (lane == 0) counts[warp] = mine;
        __syncthreads();
        n = 0;
        uint32_t to = 0;
#pragma unroll
        for (uint32_t w = 0; w < THREADS / 32; ++w) {
            if (w == warp) to = n;
            n += counts[w];
        }
#pragma unroll
        for (uint32_t k = 0; k < PER_LANE; ++k) {
            if (takes[k] >> lane & 1) list[to + __popc(takes[k] & ((1u << lane) - 1))] = e[k];
            to += __popc(takes[k]);
        }
        __syncthreads();
        const uint64_t halves = (uint64_t)n * 2 * p.n_layers;
        const uint32_t agents = p.width * AGENTS;
        piece = (uint32_t)min(p.block_bytes, (uint64_t)STAGE);
        while (piece > LEAST && halves * ((p.block_bytes + piece - 1) / piece) < agents) piece = (piece / 2 + 15) & ~15u;
        parts = (uint32_t)((p.block_bytes + piece - 1) / piece);
        pieces = halves * parts;
        per = (uint32_t)min((uint64_t)min(32u, STAGE / piece), (pieces + agents - 1) / agents);
    };
    auto take = [&]() {                         // the units of `ticket`
        const uint32_t r = ticket / a_round;
        if (r != round) {
            round = r;
            if (r * LIST < n_pairs) list_pairs(r * LIST);
            else pieces = 0;
        }
        ticket_units(per ? (pieces + per - 1) / per : 0, ticket % a_round, p.width, p.levels, at, end);
    };
    auto answered = [&]() { return (bool)__all_sync(0xffffffffu, !asks || mbar_try_wait(full + 8 * (n_tickets % SLOTS), n_tickets / SLOTS & 1)); };
    auto next_ticket = [&]() {                  // false: there are no more
        if (!asks) return open = false;
        const uint32_t slot = n_tickets % SLOTS;
        bool there = mbar_wait_bounded(full + 8 * slot, n_tickets / SLOTS & 1);
        if (!__all_sync(0xffffffffu, there)) {
            give_up();
            return false;
        }
        const bool got = answer(base + OFF_SLOT + 16 * slot, ticket);
        fence_proxy_async();                    // the answer has been read before the next one is written over it
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + 8 * slot);
        ++n_tickets;
        if (!got) {
            open = false;
            return false;
        }
        if (warp == 0) {                        // asks for the next ticket, where the slot's last answer has been read by all
            const uint32_t s = n_tickets % SLOTS;
            there = n_tickets < SLOTS || mbar_wait_bounded(empty + 8 * s, (n_tickets / SLOTS - 1) & 1);
            if (!__all_sync(0xffffffffu, there)) {
                give_up();
                return false;
            }
            if (lane == 0) {                    // (all have left the ticket that lies 2 SLOTS back)
                claims[(n_tickets + 1) & (2 * SLOTS - 1)] = 0;
                ask(base + OFF_SLOT + 16 * s, full + 8 * s);
            }
        }
        take();
        return true;
    };
    take();
    if (warp >= AGENTS) {
        // Scales: with the first piece of a block, a lane a float; the warps take the ticket's units in turn.
        do {
            for (at += (warp - AGENTS) * p.width; p.scales && at < end; at += (THREADS / 32 - AGENTS) * p.width) {
                const uint64_t first = (at * per + parts - 1) / parts, blocks = (min((at + 1) * per, pieces) + parts - 1) / parts - first;
                for (uint64_t i = lane; i < blocks * p.n_kv_heads; i += 32) {
                    const uint64_t b = first + i / p.n_kv_heads;
                    const uint32_t h = (uint32_t)(i % p.n_kv_heads);
                    const int2 e = list[b / 2 % n];
                    const LayerBytes &l = p.layer[b / 2 / n];
                    float *x = b % 2 ? l.v_scale : l.k_scale;
                    if (x && (uint32_t)e.x < l.n_blocks && (uint32_t)e.y < l.n_blocks)
                        x[(uint64_t)(uint32_t)e.y * l.scale_row + h] = x[(uint64_t)(uint32_t)e.x * l.scale_row + h];
                }
            }
        } while (next_ticket());
        if (p.scales) __threadfence();
    } else {
        unsigned long long *to = reinterpret_cast<unsigned long long *>(smem + OFF_TO) + warp * STAGES * 32 + lane;
        uint32_t *bytes = reinterpret_cast<uint32_t *>(smem + OFF_BYTES) + warp * STAGES * 32 + lane;
        const uint32_t ring = base + warp * STAGES * STAGE;
        uint32_t offset[STAGES];                // of the lane's piece in a stage: rounds may cut blocks differently
        // Issues the loads of this agent's next unit, the ticket's first that no agent has taken, into a stage; false: there is none,
        // or none yet and the loads in flight want to be seen to.
        auto issue = [&](uint32_t stage, bool others) {
            uint64_t unit = 0;
            while (open) {
                uint32_t k = lane == 0 ? atomicAdd(claims + (n_tickets & (2 * SLOTS - 1)), 1) : 0;
                unit = at + (uint64_t)__shfl_sync(0xffffffffu, k, 0) * p.width;
                if (unit < end) break;
                if (others && !answered()) return false;
                if (!next_ticket()) break;
            }
            if (!open) return false;
            const uint64_t i = unit * per + lane;
            uint32_t size = 0;
            unsigned long long src = 0;
            if (lane < per && i < pieces) {
                const uint32_t part = (uint32_t)(i % parts);
                const uint64_t h = i / parts;
                const LayerBytes &l = p.layer[h / 2 / n];
                const int2 e = list[h / 2 % n];
                if ((uint32_t)e.x < l.n_blocks && (uint32_t)e.y < l.n_blocks) {
                    const uint64_t from = (h % 2 ? l.v_base : l.k_base) + (uint64_t)part * piece;
                    size = (uint32_t)min((uint64_t)piece, p.block_bytes - (uint64_t)part * piece);
                    src = from + (uint32_t)e.x * l.block_stride;
                    to[stage * 32] = from + (uint32_t)e.y * l.block_stride;
                } else {
                    if (p.status) atomicCAS(p.status, TUTTI_OK, TUTTI_EFAULT);
                }
            }
            bytes[stage * 32] = size;
            const uint32_t all = __reduce_add_sync(0xffffffffu, size);
            const uint32_t o = ring + stage * STAGE + lane * piece;
#pragma unroll
            for (uint32_t k = 0; k < STAGES; ++k)
                if (k == stage) offset[k] = o;
            if (lane == 0) mbar_expect_tx(bars + 8 * stage, all);
            __syncwarp();
            if (size) bulk_g2s(o, src, size, bars + 8 * stage);
            return true;
        };
        uint32_t in_flight = 0, phases = 0, stage = 0;
        while (true) {
            // the stage that is filled has been read: at most the last store's may not have been
            while (in_flight < STAGES - 1 && issue((stage + in_flight) % STAGES, in_flight > 0)) ++in_flight;
            if (!in_flight) break;
            const bool there = mbar_wait_bounded(bars + 8 * stage, phases >> stage & 1);
            if (!__all_sync(0xffffffffu, there)) {
                give_up();
                // copies in flight: as long again for each
                for (uint32_t k = 0, s = stage; k < in_flight; ++k, s = s + 1 == STAGES ? 0 : s + 1) (void)mbar_wait_bounded(bars + 8 * s, phases >> s & 1);
                break;
            }
            phases ^= 1u << stage;
            uint32_t o = 0;
#pragma unroll
            for (uint32_t k = 0; k < STAGES; ++k)
                if (k == stage) o = offset[k];
            if (const uint32_t size = bytes[stage * 32]) bulk_s2g(to[stage * 32], o, size);
            bulk_commit();
            --in_flight;
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            bulk_wait_read_1();
            __syncwarp();
        }
        bulk_wait_all();                        // the copies have been written, not only read
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
        p.width = (uint32_t)tutti_ctx_sms_(ctx);
        p.levels = 1;
        // (a ticket costs a CTA 0.5 us, also where *n_pairs leaves nothing of a round)
        const uint32_t rounds = (max_pairs + LIST - 1) / LIST, most = rounds * 2 < MOST_LEVELS ? MOST_LEVELS / rounds : 2;
        // Halved as long as the last tickets have LAST_TICKET bytes, if all pairs of a round count; not for a few us of work.
        uint64_t share = 2 * p.block_bytes * p.n_layers * (max_pairs < LIST ? max_pairs : LIST) / p.width;
        for (share = share < 16 * LAST_TICKET ? 0 : share; share > LAST_TICKET && p.levels < most; share = share * 3 / 5) ++p.levels;
        const cudaError_t e = launch_behind(copy_blocks_kernel, rounds * p.levels * p.width, THREADS, SMEM, (cudaStream_t)stream, p);
        if (e != cudaSuccess) return fail(e, "copy launch");
    }
    return TUTTI_OK;
}

}  // extern "C"
