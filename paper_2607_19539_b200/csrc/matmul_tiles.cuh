// Shared by the products whose rows may be grouped by expert: where experts' rows and tiles begin, the waits and what follows one that
// gives up, tensor maps, and the body of a persistent kernel that loads, multiplies and finishes tiles in three roles.
#pragma once

#include <atomic>

#include "opcommon.cuh"
#include "ptx.cuh"

namespace moe_ovl {

enum : long long { SITE_TILE_EMPTY = 32, SITE_TILE_FULL, SITE_TILE_DONE };

constexpr int TILE_CHANNELS = 128;           // matrix instruction rows per CTA
constexpr int STAGE_ROW = 128;               // bytes of K per pipeline stage and row: one row of the 128-byte swizzle
constexpr int TILE_GROUP = 16;               // token tiles that are worked on side by side, see TileSchedule
constexpr unsigned long long TILE_TIMEOUT_NS = 2000000000ull;

// Inclusive sums over the lanes, none above `limit` (< 2^31; nor is v).  A loop, not unrolled: this runs once, before anything else
// can, and every line of its code is fetched from memory then.
__device__ __forceinline__ unsigned scan_up_to(unsigned v, unsigned limit, int lane)
{
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned w = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v = min(v + w, limit);
    }
    return v;
}

// Rows of 32 experts from e0 on, one per lane: where each one's rows begin and end, given the rows before.  Counts are cut
// so that no expert reaches beyond the rows there are.
__device__ __forceinline__ void expert_rows(int count, unsigned limit, unsigned before, int lane, unsigned &first, unsigned &last)
{
    last = min(before + scan_up_to(min((unsigned)max(count, 0), limit), limit, lane), limit);
    first = __shfl_up_sync(0xffffffffu, last, 1);
    if (lane == 0) first = before;
}
template <typename P> __device__ __forceinline__ int count_of(const P &p, int e) { return p.counts && e < p.experts ? p.counts[e] : 0; }

// Takes bytes off what the phase still waits for, as a copy of that size would.
__device__ __forceinline__ void mbar_complete_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void st_shared_cluster_u32(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// A wait that gives up, in whichever warp, leaves tile copies and matrix instructions under way: they have to land before the CTA's shared and
// tensor memory go to somebody else.  This wait has a limit of its own, which neither a caller's short one nor an aborted status shortens.
constexpr unsigned long long LANDING_NS = 2000000000ull;
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity, unsigned long long since)
{
    while (!mbar_try_wait(bar, parity) && globaltimer_ns() - since < LANDING_NS) {}
}

// mbar_wait in two parts: most of a pipeline's waits are over when they begin, and what else there is to a wait (its clock above all, which takes longer to
// read than they last) stays out of the loops.
template <typename P> __device__ __noinline__ bool long_wait(uint32_t bar, uint32_t parity, const P &p, long long site, long long index)
{
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait(bar, parity, p, site, index);
}

// A whole warp's wait, by all of its lanes alike: a branch for one of them and passing on what it has seen takes longer than the wait mostly does
// (the block product of 7919 x 28672 x 4096, a wait per 128 columns and 128 of K: 901 us with one lane's polls, 861 with all).
template <typename P> __device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const P &p, long long site, long long index)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return __all_sync(0xffffffffu, long_wait(bar, parity, p, site, index));
}

// Order of the tiles: experts one after the other; inside an expert up to TILE_GROUP token tiles form a group, and for each tile
// of channels all token tiles of the group come next to each other.  The CTAs that run side by side then share one
// tile of weights in L2, and the weights are read from HBM once per group (4096 tokens of the largest tiles).  Every worker (a
// CTA or a pair) takes every workers-th tile, so a role only ever moves forward through the experts.
template <int CHANNELS, int TOKENS> struct TileSchedule {
    const int *tile_start, *row_start;       // [experts + 1] token tiles and rows before each expert, in shared memory
    int row_tiles, expert = 0;
    struct Tile { int expert, channel0, row0, rows; };
    __device__ long long total(int experts) const { return (long long)tile_start[experts] * row_tiles; }
    __device__ Tile at(long long index)
    {
        while (index >= (long long)tile_start[expert + 1] * row_tiles) ++expert;
        const int tiles = tile_start[expert + 1] - tile_start[expert];
        const int i = (int)(index - (long long)tile_start[expert] * row_tiles);
        const int group = i / (TILE_GROUP * row_tiles), first = group * TILE_GROUP, wide = min(TILE_GROUP, tiles - first);
        const int j = i - group * TILE_GROUP * row_tiles;
        const int row0 = row_start[expert] + (first + j % wide) * TOKENS;
        return {expert, j / wide * CHANNELS, row0, min(TOKENS, row_start[expert + 1] - row0)};
    }
};

// One warp fills the schedule's tables.  `count`: count_of(lane), asked for early.
template <int TOKENS, typename P> __device__ __forceinline__ void fill_schedule(const P &p, int *tile_start, int *row_start, int count, int lane)
{
    unsigned rows_before = 0, tiles_before = 0;
    if (lane == 0) tile_start[0] = row_start[0] = 0;
    if (!p.counts && lane == 0) tile_start[1] = (p.rows - 1) / TOKENS + 1, row_start[1] = p.rows;
    const int experts = p.counts ? p.experts : 0;
#pragma unroll 1
    for (int e0 = 0; e0 < experts; e0 += 32) {
        const int e = e0 + lane;
        unsigned first, last;
        expert_rows(e0 == 0 ? count : count_of(p, e), (unsigned)p.rows, rows_before, lane, first, last);
        const unsigned tiles = tiles_before + scan_up_to((last - first + TOKENS - 1) / TOKENS, 0x7fffffffu, lane);
        if (e < experts) {
            tile_start[e + 1] = (int)tiles;
            row_start[e + 1] = (int)last;
        }
        tiles_before = __shfl_sync(0xffffffffu, tiles, 31);
        rows_before = __shfl_sync(0xffffffffu, last, 31);
    }
    __syncwarp();
}

// What one elected lane does of a warp that runs the same code in all of them: the instruction is predicated (`on`: in the elected lane), and its operands are made by
// all lanes alike, in uniform registers.  Behind a branch for one lane they would have to be gathered from that lane, which takes longer than the rest of a step.

// Tile loads of two and three dimensions, into this CTA's shared memory, counted on its barrier or (CTAS == 2) on one that may be the peer's.
template <int CTAS> __device__ __forceinline__ void load_2d(uint32_t on, uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    if constexpr (CTAS == 1)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n\t}"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(on)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n\t}"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(on)
            : "memory");
}
template <int CTAS> __device__ __forceinline__ void load_3d(uint32_t on, uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    if constexpr (CTAS == 1)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
            "@q cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(on)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
            "@q cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(on)
            : "memory");
}
__device__ __forceinline__ void expect_bytes(uint32_t on, uint32_t bar, uint32_t bytes)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
        "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}"
        ::"r"(bar), "r"(bytes), "r"(on)
        : "memory");
}

// D[tmem] (+)= A[smem] * B[smem] with 32-bit sums, by this CTA or by the CTA pair: 16-bit floats, K = 16, or 8-bit floats, K = 32.
#define MOE_OVL_UMMA(GROUP, KIND)                                                                                                   \
    asm volatile(                                                                                                                   \
        "{\n\t.reg .pred p, q;\n\t"                                                                                                 \
        "setp.ne.b32 p, %4, 0;\n\t"                                                                                                 \
        "setp.ne.b32 q, %5, 0;\n\t"                                                                                                 \
        "@q tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, p;\n\t}"                                              \
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on)                                               \
        : "memory")
template <int CTAS> __device__ __forceinline__ void umma_f16(uint32_t on, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (CTAS == 1) MOE_OVL_UMMA("1", "f16");
    else MOE_OVL_UMMA("2", "f16");
}
template <int CTAS> __device__ __forceinline__ void umma_f8(uint32_t on, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (CTAS == 1) MOE_OVL_UMMA("1", "f8f6f4");
    else MOE_OVL_UMMA("2", "f8f6f4");
}
#undef MOE_OVL_UMMA
// One arrival, in both CTAs of a pair, when every matrix instruction issued so far by this thread has finished.
template <int CTAS> __device__ __forceinline__ void commit(uint32_t on, uint32_t bar)
{
    if constexpr (CTAS == 1)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
            "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
            ::"r"(bar), "r"(on)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
            "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
            ::"r"(bar), "h"((uint16_t)3), "r"(on)
            : "memory");
}

// 32 lanes x 8 columns, and the wait for values asked of tensor memory; they are operands of the wait so that no use of them can move in front of it.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&v)[8])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                   "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

__device__ __forceinline__ float4 ld_shared_cluster_f32x4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// ------------------------------------------------------------------ persistent tiles in three roles

// CTAS CTAs (one, or a pair that shares every matrix instruction) work on a tile; STAGE_BYTES are one CTA's operands of one step of K.  ACCS accumulators of
// ACC_COLS columns of tensor memory go round.  Every SEGMENT steps have PARTS of them, side by side in the tile, which a share of the finishing warps each adds up.  TURNS > 1: that many groups of them take the accumulators in turn.
template <int CTAS_, int STAGE_BYTES_, int SMEM_BYTES_, int ACCS_, int ACC_COLS_, int FINISHERS_, int SEGMENT_, int PARTS_ = 1, int TURNS_ = 1> struct TileShape {
    static constexpr int CTAS = CTAS_, STAGE_BYTES = STAGE_BYTES_, ACCS = ACCS_, ACC_COLS = ACC_COLS_, FINISHERS = FINISHERS_, SEGMENT = SEGMENT_, PARTS = PARTS_, GROUPS = PARTS_ * TURNS_;
    static constexpr int STAGES = SMEM_BYTES_ / STAGE_BYTES_;
    static constexpr int CONTROL = 2, THREADS = 32 * (CONTROL + FINISHERS);      // the load and the matrix warp
    static constexpr int SMEM = STAGES * STAGE_BYTES + 1024;
    static_assert(ACCS * ACC_COLS <= 512 && ACC_COLS >= 32 && ACCS % GROUPS == 0 && FINISHERS % GROUPS == 0 && SEGMENT > 0, "tensor memory");
};

// Arrival of a reader of tensor memory, on a barrier that may be the peer CTA's.  What it gives back has been read (tcgen05.wait, and the fence
// in front of it) and nothing was written, so it needs no release of memory at cluster scope, which would wait for the warp's loads and stores.
__device__ __forceinline__ void arrive_read(uint32_t on, uint32_t cluster_bar)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
        "@q mbarrier.arrive.shared::cluster.b64 _, [%0];\n\t}"
        ::"r"(cluster_bar), "r"(on)
        : "memory");
}

// A finishing warp's way through the accumulators of its group.
template <typename Shape> struct Accumulators {
    uint32_t bar_full, lead_empty, tmem;
    int lane, group = 0, acc = 0;
    uint32_t phase = 0;
    bool there = false;                      // this lane has seen what wait() would wait for
    template <typename P> __device__ __forceinline__ bool wait(const P &p, long long index)
    {
        const bool ok = __all_sync(0xffffffffu, there) || warp_wait(bar_full + 8 * acc, phase, p, SITE_TILE_DONE, index);
        there = false;
        tc_fence_after();
        return ok;
    }
    // A look at the next one ahead of its wait, for whoever has something else to do meanwhile; behind release().
    __device__ __forceinline__ void look() { there = mbar_test_wait(bar_full + 8 * acc, phase); }
    __device__ __forceinline__ uint32_t columns() const { return tmem + (uint32_t)(acc * Shape::ACC_COLS); }
    __device__ __forceinline__ void release()
    {
        tc_fence_before();
        __syncwarp();
        arrive_read(lane == 0, lead_empty + 8 * acc);
        if ((acc += Shape::GROUPS) >= Shape::ACCS) acc = group, phase ^= 1u;
    }
};

// After a give-up: waits for the copies that are under way, by one thread of the CTA whose barriers count them.  `mine`, `peers`: stages that
// this CTA and (in a pair) the other one have issued; they are at most a ring apart, since neither refills a stage that the other has
// not filled.  A fill of one side alone counts that side's bytes alone: the other side's are taken off, or, where this CTA's thread has not
// announced the fill, half of the usual number is announced.
template <typename Shape> __device__ void await_copies(uint32_t bar_full, uint32_t mine, uint32_t peers)
{
    constexpr uint32_t STAGES = Shape::STAGES;
    const uint32_t last = Shape::CTAS == 1 ? mine : max(mine, peers);
    const unsigned long long t0 = globaltimer_ns();
    for (uint32_t i = last > STAGES ? last - STAGES : 0; i < last; ++i) {
        const uint32_t bar = bar_full + 8 * (i % STAGES);
        if (Shape::CTAS == 2 && i >= peers) mbar_complete_tx(bar, Shape::STAGE_BYTES);
        else if (Shape::CTAS == 2 && i >= mine) mbar_arrive_expect_tx(bar, Shape::STAGE_BYTES);
        drain(bar, (i / STAGES) & 1u, t0);
    }
}

// Body of a persistent kernel: one load warp, one warp that issues the matrix instructions, FINISHERS warps that read the
// accumulators.  Each role walks the same tiles.  The whole of a load or matrix warp runs its loop, with everything the same in all lanes, and one
// elected lane issues: copies and matrix instructions take their operands from uniform registers.
// `Work` says what a tile is: begin(lane) fills the tables, by one warp; total(); at(t); steps(tile) of K, 0 for a tile that nothing is loaded for;
// load(on, tile's operands, shared address, barrier, step); instruction(tile); multiply(on, accumulator, stage's address / 16, instruction, first, part);
// finish(tile, accumulators, warp, lane), false when a wait gave up; close(lane), when a finishing warp has done its last tile.  With SPLITS > 1 a cluster of that many CTAs works on one tile, each on its `split` of the steps; finish()
// leaves the part in shared memory and join(tile), called by all threads when the parts of all are there, adds them up.
template <typename Work, typename P> __device__ __forceinline__ void run_tiles(Work work, const P &p, uint8_t *smem_raw)
{
    using Shape = typename Work::Shape;
    constexpr int CTAS = Shape::CTAS, STAGES = Shape::STAGES, ACCS = Shape::ACCS;
    __shared__ __align__(8) uint64_t s_bars[2 * STAGES + 2 * ACCS + 1];
    __shared__ uint32_t s_tmem;
    __shared__ uint32_t s_gave_up, s_issued[2];      // a wait for operands or room ran out, here or in the peer; rank 0: stages that each CTA has issued
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t operands16 = (smem_base & 0x3ffffu) / 16;         // in a cluster the address has the CTA's place above these bits
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * STAGES;
    const uint32_t bar_tfull = bar_empty + 8 * STAGES, bar_tempty = bar_tfull + 8 * ACCS, bar_drain = bar_tempty + 8 * ACCS;
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    // alone, one of a pair, or one of Work::SPLITS that share a tile's steps
    static_assert(CTAS == 1 || Work::SPLITS == 1, "pairs do not share steps");
    const uint32_t place = CTAS * Work::SPLITS == 1 ? 0 : cluster_ctarank(), rank = CTAS == 1 ? 0 : place;
    const uint32_t lead_full = CTAS == 1 ? bar_full : map_to_cta(bar_full, 0);
    const uint32_t lead_tempty = CTAS == 1 ? bar_tempty : map_to_cta(bar_tempty, 0);
    const long long first = blockIdx.x / (CTAS * Work::SPLITS), step = gridDim.x / (CTAS * Work::SPLITS);
    work.rank = (int)rank;
    if constexpr (Work::SPLITS > 1) work.split = (int)place;
    bool ok = true;
    auto gave_up = [&]() {
        s_gave_up = 1;
        if (CTAS == 2) st_shared_cluster_u32(map_to_cta(smem_u32(&s_gave_up), rank ^ 1u), 1);
    };

    if (warp == 0) {
        for (int i = lane; i < 2 * STAGES + 2 * ACCS + 1; i += 32)
            // full: the first CTA's load thread arrives, expecting all CTAs' bytes; accumulators empty: one arrival per finishing warp
            mbar_init(bar_full + 8 * i, i >= 2 * STAGES + ACCS && i < 2 * STAGES + 2 * ACCS ? Shape::FINISHERS / Shape::GROUPS * CTAS : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (lane == 0) s_gave_up = 0;
        __syncwarp();
        after_previous();
        work.begin(lane);
    } else if (warp == 1) {
        if (CTAS == 1) tmem_alloc_self(smem_u32(&s_tmem), ACCS * Shape::ACC_COLS);
        else tmem_alloc(smem_u32(&s_tmem), ACCS * Shape::ACC_COLS);
    }
    tc_fence_before();
    after_previous();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();
    may_follow();
    tc_fence_after();
    const uint32_t tmem = uniform(s_tmem);
    const long long total = work.total();
    if (warp >= Shape::CONTROL) {
        const int group = (warp - Shape::CONTROL) / (Shape::FINISHERS / Shape::GROUPS);
        Accumulators<Shape> accs{bar_tfull, lead_tempty, tmem, lane, group, group};
        for (long long t = first; t < total; t += step)
            if (!work.finish(work.at(t), accs, p, warp - Shape::CONTROL, lane)) break;         // a warp leaves the loop as one
        __syncwarp();
        work.close(lane);
    } else if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0, issued = 0;
        if (!p.no_loads) {
            const uint32_t leader = elect_one(), announces = leader && rank == 0;
            for (long long t = first; ok && t < total; t += step) {
                const auto tile = work.at(t);
                const auto from = work.operands(tile, leader);
                const int steps = uniform(work.steps(tile));
                int k = 0;
                for (; k < steps; ++k) {
                    ok = warp_wait(bar_empty + 8 * stage, phase ^ 1u, p, SITE_TILE_EMPTY, t);
                    if (!ok) break;
                    expect_bytes(announces, bar_full + 8 * stage, CTAS * Shape::STAGE_BYTES);
                    work.load(leader, from, smem_base + stage * Shape::STAGE_BYTES, lead_full + 8 * stage, k);
                    if (++stage == STAGES) stage = 0, phase ^= 1u;
                }
                issued += (uint32_t)k;
            }
        }
        __syncwarp();
        if (lane == 0) {
            if (rank == 0) s_issued[0] = issued;
            else st_shared_cluster_u32(map_to_cta(smem_u32(&s_issued[1]), 0), issued);
            if (!ok) gave_up();
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t leader = elect_one();
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            for (long long t = first; ok && t < total; t += step) {
                const auto tile = work.at(t);
                const uint32_t idesc = uniform(work.instruction(tile));
                const int steps = uniform(work.steps(tile));
                for (int k = 0; k < steps; ++k) {
                    const bool begins = k % Shape::SEGMENT == 0, ends = k == steps - 1 || k % Shape::SEGMENT == Shape::SEGMENT - 1;
                    ok = warp_wait(bar_full + 8 * stage, phase, p, SITE_TILE_FULL, k);
                    if (!ok) break;
#pragma unroll
                    for (int part = 0; part < Shape::PARTS; ++part) {
                        if (begins) ok = ok && warp_wait(bar_tempty + 8 * acc, acc_phase ^ 1u, p, SITE_TILE_DONE, t);
                        if (!ok) break;
                        tc_fence_after();
                        work.multiply(leader, tmem + (uint32_t)(acc * Shape::ACC_COLS), operands16 + (uint32_t)stage * (Shape::STAGE_BYTES / 16), idesc, begins, part);
                        if (ends) commit<CTAS>(leader, bar_tfull + 8 * acc);
                        if (ends && ++acc == ACCS) acc = 0, acc_phase ^= 1u;
                    }
                    if (!ok) break;
                    commit<CTAS>(leader, bar_empty + 8 * stage);
                    if (++stage == STAGES) stage = 0, phase ^= 1u;
                }
            }
            if (leader) {
                if (CTAS == 1) umma_commit_one(bar_drain);      // every MMA has finished before tensor memory goes
                else if (ok) umma_commit_self(bar_drain);       // the peer has waited for its last accumulator, and does not wait for this
                else umma_commit_pair(bar_drain);
            }
            drain(bar_drain, 0, globaltimer_ns());
            if (!ok && lane == 0) gave_up();
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();          // the peer no longer signals this CTA's barriers or reads its operands
    if constexpr (Work::SPLITS > 1) {
        cluster_sync_all();                     // the parts are in everybody's shared memory
        if (first < total) work.join(work.at(first));
        __syncwarp();
        cluster_sync_all();                     // and stay until everybody has read them
    }
    if (s_gave_up) {
        // but copies may be under way, which rank 0's barriers count for both, and matrix instructions' signals to rank 1
        if (threadIdx.x == 0) {
            if (rank == 0) await_copies<Shape>(bar_full, s_issued[0], s_issued[CTAS - 1]);
            else drain(bar_drain, 0, globaltimer_ns());
        }
        __syncthreads();
        if (CTAS == 2) cluster_sync_all();
    }
    tc_fence_after();
    if (warp == 1) {
        if (CTAS == 1) tmem_dealloc_self(tmem, ACCS * Shape::ACC_COLS);
        else tmem_dealloc(tmem, ACCS * Shape::ACC_COLS);
    }
}

// The output of a tile whose steps a cluster has shared: a warp adds up the parts of a row, four columns per lane, SPLITS loads in flight.  The CTAs and their warps take the
// rows in turn.  part: [rows][PITCH] in shared memory, at the same place in every CTA; out: the tile's first row.
template <int SPLITS, int PITCH = TILE_CHANNELS, typename Out>
__device__ __forceinline__ void join_parts(const float *part, Out *out, long long stride, int channel0, int n, int rows, int split, bool accumulate)
{
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, ch = channel0 + 4 * lane;
    for (int j = split + SPLITS * warp; j < rows; j += SPLITS * (blockDim.x / 32)) {
        float4 v[SPLITS];
#pragma unroll
        for (int s = 0; s < SPLITS; ++s) v[s] = ld_shared_cluster_f32x4(map_to_cta(smem_u32(part + j * PITCH + 4 * lane), (uint32_t)s));
        float sum[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
        for (int s = 1; s < SPLITS; ++s) sum[0] += v[s].x, sum[1] += v[s].y, sum[2] += v[s].z, sum[3] += v[s].w;
        Out *at = out + (long long)j * stride + ch;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((unsigned)(ch + i) < (unsigned)n) at[i] = from_f32<Out>(accumulate ? sum[i] + to_f32(at[i]) : sum[i]);
    }
}

// ------------------------------------------------------------------ host

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn()
{
    static std::atomic<EncodeTiledFn> known{nullptr};
    EncodeTiledFn f = known.load(std::memory_order_acquire);
    if (f) return f;
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult res;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &res) != cudaSuccess || res != cudaDriverEntryPointSuccess)
        return nullptr;
    f = reinterpret_cast<EncodeTiledFn>(fn);
    known.store(f, std::memory_order_release);
    return f;
}

// `depth` matrices (0: one, in a map of two dimensions) of `rows` rows of `cols` elements; rows lie `stride` bytes apart, matrices `far` bytes.
// Boxes of 128 bytes x box_rows rows with the 128-byte swizzle; what lies beyond a matrix is read as 0.
inline bool encode_tiles(CUtensorMap *map, CUtensorMapDataType type, int element, const void *base, long long cols, long long rows, long long stride,
                         int depth, long long far, int box_rows)
{
    const EncodeTiledFn f = encode_fn();
    if (!f) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
    const cuuint64_t strides[2] = {(cuuint64_t)stride, (cuuint64_t)far};
    const cuuint32_t box[3] = {(cuuint32_t)(STAGE_ROW / element), (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
    return f(map, type, depth ? 3 : 2, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Allows a kernel its dynamic shared memory, once per device.
template <typename K> bool allow_smem(K kernel, int bytes, int device, std::atomic<unsigned long long> &done)
{
    const unsigned long long bit = device < 64 ? 1ull << device : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

inline int sm_count(int device)
{
    static std::atomic<int> known[64];
    if (device >= 64) return 148;
    int n = known[device].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 2) return 2;
        known[device].store(n, std::memory_order_relaxed);
    }
    return n;
}

// How many CTAs share a tile's steps of K: as many as there are clusters of on the device at once (a second wave costs more than sharing gains), four steps for each at least.  A step
// takes a CTA `step_ns` ns; sharing costs about 1.2 us, and 0.03 us per row of the tile, whose parts have to be added up.  Measured, us: 1 row, n = 512, k = 4096 12.1 unshared, 5.2 with
// eight; 64 rows 11.9 and 6.4; n = k = 4096, 1 row 12.4 and 6.6 with four; 64 rows, n = 512, k = 1024 4.9 and 5.6.
inline int splits_of(long long tiles, int per_sm, long long steps, int rows, int step_ns)
{
    const int clusters[3] = {74 * per_sm, per_sm == 2 ? 71 : 33, per_sm == 2 ? 33 : 15};     // of 2, 4, 8 CTAs
    int s = 1;
    for (int i = 0; i < 3 && tiles <= clusters[i] && steps >= 8 * s; ++i) s *= 2;
    return steps * (s - 1) * step_ns > s * (1200ll + 30 * rows) ? s : 1;
}

}  // namespace moe_ovl
