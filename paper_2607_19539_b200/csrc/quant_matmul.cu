// Product of 8-bit integers with a scale per token and per channel, dense or per expert (moe_ovl_quant_matmul in
// include/moe_ovl.h):  out[m][n] = (sum_k a[m][k] * b[e][n][k]) * a_scale[m] * b_scale[e][n].
//
// The operands are swapped on the tensor cores: 128 weight rows (channels) are the matrix instruction's M side and
// BN tokens its N side, because the number of tokens is what varies (one, a handful, a ragged group) and N goes in steps
// of 16 while M does not.  The accumulator then has a channel per lane and a token per column: the channel's scale is one
// register, and a warp's 32 lanes store 32 neighbouring channels of a token.  Sums are exact 32-bit integers, so splitting
// K over the CTAs of a cluster and adding their parts changes nothing.
#include <algorithm>

#include "matmul_tiles.cuh"

using namespace moe_ovl;

namespace {

constexpr int QM_ROWS = TILE_CHANNELS;       // channels per CTA
constexpr int QM_K = STAGE_ROW;              // K per pipeline stage: one 128-byte swizzle row
constexpr int QM_A_BYTES = QM_ROWS * QM_K;
constexpr int QM_THREADS = 192;              // load warp, MMA warp, 4 epilogue warps

struct QmP {
    int rows, n, k, experts;                 // experts 0: one matrix
    int row_tiles;                           // tiles of QM_ROWS channels per expert
    const int *counts;
    const float *a_scale, *b_scale;
    void *out;
    long long out_stride;
    int *status;
    unsigned long long timeout_ns;
    bool no_loads;                           // test hook
};

struct QmTile { int expert, row0, rows; };   // rows 0: beyond the last tile

// Channels of a tile end behind the last one: without sign, where they pass 2^31 too.
__device__ __forceinline__ bool has_channel(const QmP &p, int channel) { return (unsigned)channel < (unsigned)p.n; }
// The `index`-th tile of at most `height` tokens, experts in order.  One warp; every lane gets the answer.  `count`: count_of(lane).
__device__ QmTile find_tile(const QmP &p, int index, int height, int count, int lane)
{
    if (!p.counts) {
        const long long row0 = (long long)index * height;
        if (row0 >= p.rows) return {0, 0, 0};
        return {0, (int)row0, min(height, p.rows - (int)row0)};
    }
    unsigned rows_before = 0, tiles_before = 0;
#pragma unroll 1
    for (int e0 = 0; e0 < p.experts; e0 += 32) {
        unsigned first, last;
        expert_rows(e0 == 0 ? count : count_of(p, e0 + lane), (unsigned)p.rows, rows_before, lane, first, last);
        const unsigned tiles = (last - first + height - 1) / height;
        const unsigned start = tiles_before + scan_up_to(tiles, 0x7fffffffu, lane) - tiles;
        const unsigned hit = __ballot_sync(0xffffffffu, (unsigned)index >= start && (unsigned)index < start + tiles);
        if (hit) {
            const int owner = __ffs(hit) - 1;
            const int r = (int)__shfl_sync(0xffffffffu, first + (index - start) * height, owner);
            const int end = (int)__shfl_sync(0xffffffffu, last, owner);
            return {e0 + owner, r, min(height, end - r)};
        }
        tiles_before = __shfl_sync(0xffffffffu, start + tiles, 31);
        rows_before = __shfl_sync(0xffffffffu, last, 31);
    }
    return {0, 0, 0};
}

template <typename Out> __device__ __forceinline__ void store_scaled(Out *at, int sum, float a_scale, float b_scale)
{
    *at = from_f32<Out>(__int2float_rn(sum) * a_scale * b_scale);
}

// Two CTAs per SM: while one fills its pipeline or stores, the other streams.
template <int BN> struct QmShape {
    static constexpr int STAGE_BYTES = QM_A_BYTES + BN * QM_K;
    static constexpr int STAGES = 104 * 1024 / STAGE_BYTES;
    static constexpr int SMEM = STAGES * STAGE_BYTES + 1024 + 256;
};

// A whole warp's wait, polled by one lane: the others' polls would only compete with the load and MMA threads' own.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const QmP &p, long long index, int lane)
{
    bool ok = true;
    if (lane == 0) ok = mbar_wait(bar, parity, p, SITE_TILE_DONE, index);
    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
    if (ok) mbar_try_wait(bar, parity);      // done already: this lane's own look, for the order of what it reads next
    return ok;
}

// Few tiles: one tile (128 channels x BN tokens) per cluster, whose SPLITS CTAs share its K.  Each leaves its part in its shared
// memory, and the tokens are dealt out for the sum and the scaling.
template <int BN, int SPLITS, typename Out>
__global__ void __launch_bounds__(QM_THREADS)
quant_matmul_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, const QmP p)
{
    constexpr int STAGES = QmShape<BN>::STAGES, STAGE_BYTES = QmShape<BN>::STAGE_BYTES, TMEM_COLS = BN < 32 ? 32 : BN;
    extern __shared__ uint8_t smem_raw[];
    __shared__ QmTile s_tile;
    __shared__ uint32_t s_tmem, s_gave_up;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar_full = smem_base + STAGES * STAGE_BYTES, bar_empty = bar_full + 8 * STAGES, bar_done = bar_empty + 8 * STAGES;
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % SPLITS);
    const unsigned tile_index = blockIdx.x / SPLITS;
    const int row_tile = (int)(tile_index % (unsigned)p.row_tiles);

    if (warp == 0) {
        after_previous();
        const QmTile t = find_tile(p, (int)(tile_index / (unsigned)p.row_tiles), BN, count_of(p, lane), lane);
        if (lane == 0) s_tile = t;
    } else if (warp == 1) {
        tmem_alloc_self(smem_u32(&s_tmem), TMEM_COLS);
    } else if (threadIdx.x == 64) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(bar_full + 8 * i, 1);
            mbar_init(bar_empty + 8 * i, 1);
        }
        mbar_init(bar_done, 1);
        s_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    after_previous();
    __syncthreads();
    may_follow();
    tc_fence_after();
    const QmTile tile = {uniform(s_tile.expert), uniform(s_tile.row0), uniform(s_tile.rows)};
    const uint32_t tmem = uniform(s_tmem);
    const int steps_all = (p.k + QM_K - 1) / QM_K;
    const int k0 = steps_all * rank / SPLITS, k1 = steps_all * (rank + 1) / SPLITS;
    int issued = 0;                         // warp 0: stages
    if (tile.rows > 0) {
        if (warp == 0 && !p.no_loads) {
            const bool leader = elect_one();
            const int y_b = tile.expert * p.n + row_tile * QM_ROWS;
            int stage = 0;
            uint32_t phase = 0;
            for (int k = k0; k < k1; ++k, ++issued) {
                if (!__all_sync(0xffffffffu, mbar_wait(bar_empty + 8 * stage, phase ^ 1u, p, SITE_TILE_EMPTY, k))) break;
                const uint32_t sa = smem_base + stage * STAGE_BYTES;
                if (leader) {
                    mbar_arrive_expect_tx(bar_full + 8 * stage, STAGE_BYTES);
                    tma_load_2d_self(sa, &map_b, bar_full + 8 * stage, k * QM_K, y_b);
                    tma_load_2d_self(sa + QM_A_BYTES, &map_a, bar_full + 8 * stage, k * QM_K, tile.row0);
                }
                if (++stage == STAGES) stage = 0, phase ^= 1u;
            }
            if (issued < k1 - k0) s_gave_up = 1;
        } else if (warp == 1) {
            const bool leader = elect_one();
            int stage = 0;
            uint32_t phase = 0;
            for (int k = k0; k < k1; ++k) {
                if (!__all_sync(0xffffffffu, mbar_wait(bar_full + 8 * stage, phase, p, SITE_TILE_FULL, k))) {
                    s_gave_up = 1;
                    break;
                }
                tc_fence_after();
                const uint32_t sa = smem_base + stage * STAGE_BYTES;
                if (leader) {
                    const uint64_t da = umma_smem_desc(sa), db = umma_smem_desc(sa + QM_A_BYTES);
#pragma unroll
                    for (int i = 0; i < QM_K / 32; ++i)
                        umma_i8<1>(tmem, da + (uint64_t)(i * 2), db + (uint64_t)(i * 2), umma_idesc_i8(QM_ROWS, BN), (k > k0 || i > 0) ? 1u : 0u);
                    umma_commit_one(bar_empty + 8 * stage);
                }
                if (++stage == STAGES) stage = 0, phase ^= 1u;
            }
            if (leader) umma_commit_one(bar_done);
        }
    }
    __syncwarp();
    // scales of this lane's channel and of tokens `lane`, `lane` + 32, ..: here before they are needed
    const int own = (warp - 2) * 32 + lane, ch = row_tile * QM_ROWS + own;
    const bool in = has_channel(p, ch);
    float b_scale = 0.0f, a_scale[(BN + 31) / 32] = {};
    if (tile.rows > 0 && warp >= 2) {
        if (in) b_scale = p.b_scale[(long long)tile.expert * p.n + ch];
#pragma unroll
        for (int i = 0; i < (BN + 31) / 32; ++i)
            if (i * 32 + lane < tile.rows) a_scale[i] = p.a_scale[tile.row0 + i * 32 + lane];
    }
    if (tile.rows > 0) {
        // everybody waits: nothing of the pipeline is in use behind this point, and its memory can hold the parts
        if (!warp_wait(bar_done, 0, p, tile.row0, lane)) s_gave_up = 1;
        tc_fence_after();
    }
    if (tile.rows > 0 && warp >= 2) {
        const int quarter = warp & 3;                       // a warp reads the lanes of its position among four
        const int c = quarter * 32 + lane;
        for (int t0 = 0; t0 < BN && t0 < tile.rows; t0 += 16) {
            uint32_t v[16];
            tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + t0, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j)
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(smem_base + 4u * (uint32_t)((t0 + j) * QM_ROWS + c)), "r"(v[j]) : "memory");
        }
    }
    __syncwarp();
    cluster_sync_all();
    if (tile.rows > 0 && warp >= 2) {
        // the parts of two tokens at a time: 2 * SPLITS loads in flight
        for (int t = 2 * rank; t < tile.rows; t += 2 * SPLITS) {
            uint32_t part[2][SPLITS];
            const bool two = t + 1 < tile.rows;
#pragma unroll
            for (int s = 0; s < SPLITS; ++s) {
                const uint32_t at = map_to_cta(smem_base + 4u * (uint32_t)(t * QM_ROWS + own), (uint32_t)s);
                part[0][s] = ld_shared_cluster_u32(at);
                part[1][s] = two ? ld_shared_cluster_u32(at + 4u * QM_ROWS) : 0u;
            }
            uint32_t sum[2] = {0, 0};
#pragma unroll
            for (int s = 0; s < SPLITS; ++s) {
                sum[0] += part[0][s];
                sum[1] += part[1][s];
            }
            float mine = a_scale[0];
#pragma unroll
            for (int i = 1; i < (BN + 31) / 32; ++i) mine = t >= 32 * i ? a_scale[i] : mine;
            const float a0 = __shfl_sync(0xffffffffu, mine, t & 31), a1 = __shfl_sync(0xffffffffu, mine, (t + 1) & 31);
            if (in) {
                Out *out = static_cast<Out *>(p.out) + (long long)(tile.row0 + t) * p.out_stride + ch;
                store_scaled(out, (int)sum[0], a0, b_scale);
                if (two) store_scaled(out + p.out_stride, (int)sum[1], a1, b_scale);
            }
        }
    }
    __syncwarp();
    cluster_sync_all();                                 // the parts stay until everybody has read them
    tc_fence_before();
    __syncthreads();
    if (s_gave_up) {
        if (threadIdx.x == 0) {
            // the last fill of every stage, and the matrix instructions
            const unsigned long long t0 = globaltimer_ns();
            for (int i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i)
                drain(bar_full + 8 * (i % STAGES), (uint32_t)(i / STAGES) & 1u, t0);
            drain(bar_done, 0, t0);
        }
        __syncthreads();
    }
    tc_fence_after();
    if (warp == 1) tmem_dealloc_self(tmem, TMEM_COLS);
}

// ------------------------------------------------------------------ enough tiles for every SM: persistent CTAs, alone or in pairs

constexpr int QP_THREADS = 320;              // load warp, MMA warp, 8 epilogue warps

// CTAS CTAs work on a tile of 128 * CTAS channels x TOKENS tokens: each holds 128 channels and its share of the tokens.  What
// is not needed for tokens deepens the pipeline: with few tokens the kernel streams weights, and the bytes in flight carry it.
template <int CTAS_, int TOKENS> struct QpShape {
    static constexpr int CTAS = CTAS_;
    static constexpr int STAGE_BYTES = QM_A_BYTES + TOKENS / CTAS * QM_K;
    static constexpr int STAGES = 200 * 1024 / STAGE_BYTES;
    static constexpr int SMEM = STAGES * STAGE_BYTES + 1024 + 512;
    static constexpr int ACC_COLS = TOKENS < 32 ? 32 : TOKENS;      // of tensor memory, per accumulator
};

// The load warp's place in its sequence of stages.  The whole warp runs the loop, with everything in it the same in all lanes, and
// one elected lane issues: tile copies take their operands from uniform registers, and where the compiler cannot tell that a
// value is uniform (one lane's branch, values out of shared memory) it gathers them anew for every copy.  The loop of the stages is kept
// short: one warp's instructions follow each other slowly, and 64-bit counters in it cost a tenth of the streaming rate.
template <int CTAS, int TOKENS> struct QpLoader {
    using Shape = QpShape<CTAS, TOKENS>;
    uint32_t smem_base, bar_full, bar_empty, lead_full;
    int rank, stage = 0;
    uint32_t phase = 0, issued = 0;          // issued: stages, all in all
    bool leader;
    // Issues stages k0 .. k1 - 1 of a tile; false: a wait gave up.  FRESH: the stages have never been used.
    template <bool FRESH>
    __device__ __forceinline__ bool run(const QmP &p, const CUtensorMap &map_b, const CUtensorMap &map_a, int y_b, int y_a, int k0, int k1)
    {
        int k = k0;
        for (; k < k1; ++k) {
            if (!FRESH && !__all_sync(0xffffffffu, mbar_wait(bar_empty + 8 * stage, phase ^ 1u, p, SITE_TILE_EMPTY, y_b))) break;
            const uint32_t sa = smem_base + stage * Shape::STAGE_BYTES;
            if (leader) {
                if (CTAS == 1) {
                    mbar_arrive_expect_tx(bar_full + 8 * stage, Shape::STAGE_BYTES);
                    tma_load_2d_self(sa, &map_b, bar_full + 8 * stage, k * QM_K, y_b);
                    tma_load_2d_self(sa + QM_A_BYTES, &map_a, bar_full + 8 * stage, k * QM_K, y_a);
                } else {
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * stage, 2 * Shape::STAGE_BYTES);
                    tma_load_2d(sa, &map_b, lead_full + 8 * stage, k * QM_K, y_b);
                    tma_load_2d(sa + QM_A_BYTES, &map_a, lead_full + 8 * stage, k * QM_K, y_a);
                }
            }
            if (++stage == Shape::STAGES) stage = 0, phase ^= 1u;
        }
        issued += (uint32_t)(k - k0);
        return k == k1;
    }
};

// Persistent, one CTA per SM.
// CTAS = 2: pairs of CTAs share every matrix instruction (cta_group::2), 256 channels x TOKENS tokens, each CTA holding
// its 128 channels and HALF of the tokens, which halves the operand bytes per SM against single CTAs -- at 8 bits the tensor
// cores eat operands as fast as at 16, and that traffic out of L2 is what would bound large products (single CTAs: 1.32 ms at 7919 x 28672 x 4096, pairs 0.58 ms).
// CTAS = 1: for few tokens, where the weights' way from HBM is all that counts: nothing waits for a second CTA, and the first
// loads are under way before the rest of the block is set up.
// Accumulators are double buffered (2 x 256 columns of tensor memory at most): a tile is scaled and stored while the next one runs.
template <int CTAS, int TOKENS, typename Out>
__global__ void __launch_bounds__(QP_THREADS, 1)
quant_matmul_tiles_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, const QmP p)
{
    using Shape = QpShape<CTAS, TOKENS>;
    constexpr int STAGES = Shape::STAGES, STAGE_BYTES = Shape::STAGE_BYTES, ACC_COLS = Shape::ACC_COLS;
    extern __shared__ uint8_t smem_raw[];
    __shared__ int s_tile_start[1025], s_row_start[1025];
    __shared__ uint32_t s_tmem;
    __shared__ uint32_t s_gave_up, s_issued[2];      // a wait for operands or room ran out, here or in the peer; rank 0: stages that each CTA has issued
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar_full = smem_base + STAGES * STAGE_BYTES, bar_empty = bar_full + 8 * STAGES;
    const uint32_t bar_tfull = bar_empty + 8 * STAGES, bar_tempty = bar_tfull + 16, bar_drain = bar_tempty + 16;
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    const uint32_t rank = CTAS == 1 ? 0 : cluster_ctarank();
    const uint32_t lead_full = CTAS == 1 ? bar_full : map_to_cta(bar_full, 0);
    const uint32_t lead_tempty = CTAS == 1 ? bar_tempty : map_to_cta(bar_tempty, 0);
    const int ksteps = (p.k + QM_K - 1) / QM_K, experts = p.experts > 0 ? p.experts : 1;
    TileSchedule<CTAS * QM_ROWS, TOKENS> sched{s_tile_start, s_row_start, (p.n - 1) / (CTAS * QM_ROWS) + 1};
    const long long first = blockIdx.x / CTAS, step = gridDim.x / CTAS;
    QpLoader<CTAS, TOKENS> loader{smem_base, bar_full, bar_empty, lead_full, (int)rank};
    int early = 0;                          // stages of the first tile that are issued before the block is set up
    bool ok = true;
    // where a tile's operands begin; a pair's CTAs hold the halves of the instruction's N side
    auto rows_of = [&](long long t, int &y_b, int &y_a) {
        const auto tile = sched.at(t);
        y_b = uniform(tile.expert * p.n + tile.channel0 + (int)rank * QM_ROWS);
        y_a = uniform(tile.row0 + (int)rank * ((tile.rows + 31) / 32 * 16));
    };

    auto gave_up = [&]() {
        s_gave_up = 1;
        if (CTAS == 2) st_shared_cluster_u32(map_to_cta(smem_u32(&s_gave_up), rank ^ 1u), 1);
    };

    if (warp == 0) {
        static_assert(STAGES <= 27, "a lane per barrier");
        if (lane < STAGES) {
            mbar_init(bar_full + 8 * lane, 1);            // the leader's load thread arrives, expecting all CTAs' bytes
            mbar_init(bar_empty + 8 * lane, 1);
        } else if (lane >= 27) {
            // lanes 27 .. 31: accumulators full, accumulators empty (one arrival per epilogue warp), drained
            const int i = lane - 27;
            mbar_init(i < 2 ? bar_tfull + 8 * i : i < 4 ? bar_tempty + 8 * (i - 2) : bar_drain, i < 2 || i == 4 ? 1 : 8 * CTAS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (lane == 0) s_gave_up = 0;
        __syncwarp();
        after_previous();
        fill_schedule<TOKENS>(p, s_tile_start, s_row_start, count_of(p, lane), lane);
        loader.leader = elect_one();
        if (CTAS == 1 && !p.no_loads && first < sched.total(experts)) {
            int y_b, y_a;
            rows_of(first, y_b, y_a);
            early = min(ksteps, STAGES);
            loader.template run<true>(p, map_b, map_a, y_b, y_a, 0, early);
        }
    } else if (warp == 1) {
        if (CTAS == 1) tmem_alloc_self(smem_u32(&s_tmem), 2 * ACC_COLS);
        else tmem_alloc(smem_u32(&s_tmem), 2 * ACC_COLS);
    }
    tc_fence_before();
    after_previous();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();
    may_follow();
    tc_fence_after();
    const uint32_t tmem = uniform(s_tmem);
    const long long total = sched.total(experts);

    if (warp == 0) {
        if (!p.no_loads) {
            for (long long t = first; ok && t < total; t += step) {
                int y_b, y_a;
                rows_of(t, y_b, y_a);
                ok = loader.template run<false>(p, map_b, map_a, y_b, y_a, early, ksteps);
                early = 0;
            }
        }
        if (lane == 0) {
            if (rank == 0) s_issued[0] = loader.issued;
            else st_shared_cluster_u32(map_to_cta(smem_u32(&s_issued[1]), 0), loader.issued);
            if (!ok) gave_up();
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            const bool leader = elect_one();
            const uint64_t desc_b = umma_smem_desc(smem_base);      // of stage 0; addresses are below 2^18, in units of 16 bytes
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            for (long long t = first; ok && t < total; t += step) {
                // fewer tokens than a full tile: a narrower instruction
                const uint32_t idesc = uniform(umma_idesc_i8(CTAS * QM_ROWS, (sched.at(t).rows + 16 * CTAS - 1) / (16 * CTAS) * (16 * CTAS)));
                ok = __all_sync(0xffffffffu, mbar_wait<CTAS == 2>(bar_tempty + 8 * acc, acc_phase ^ 1u, p, SITE_TILE_DONE, t));
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(acc * ACC_COLS);
                for (int k = 0; k < ksteps; ++k) {
                    ok = __all_sync(0xffffffffu, mbar_wait(bar_full + 8 * stage, phase, p, SITE_TILE_FULL, k));
                    if (!ok) break;
                    tc_fence_after();
                    if (leader) {
                        const uint64_t da = desc_b + (uint32_t)stage * (STAGE_BYTES / 16), db = da + QM_A_BYTES / 16;
#pragma unroll
                        for (int i = 0; i < QM_K / 32; ++i)
                            umma_i8<CTAS>(d, da + (uint64_t)(i * 2), db + (uint64_t)(i * 2), idesc, (k | i) != 0 ? 1u : 0u);
                        if (CTAS == 1) umma_commit_one(bar_empty + 8 * stage);
                        else umma_commit_pair(bar_empty + 8 * stage);
                    }
                    if (++stage == STAGES) stage = 0, phase ^= 1u;
                }
                if (!ok) break;
                if (leader) {
                    if (CTAS == 1) umma_commit_one(bar_tfull + 8 * acc);
                    else umma_commit_pair(bar_tfull + 8 * acc);
                }
                if ((acc ^= 1) == 0) acc_phase ^= 1u;
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
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;          // lanes 32 * quarter .., every other 32 columns
        int acc = 0;
        uint32_t acc_phase = 0;
        for (long long t = first; t < total; t += step) {
            const auto tile = sched.at(t);
            const int ch = tile.channel0 + (int)rank * QM_ROWS + quarter * 32 + lane;
            const bool in = has_channel(p, ch);
            const float bs = in ? p.b_scale[(long long)tile.expert * p.n + ch] : 0.0f;
            // a warp leaves the loop as one: what follows needs all of its lanes
            if (!warp_wait(bar_tfull + 8 * acc, acc_phase, p, t, lane)) break;
            tc_fence_after();
            for (int c = half * 32; c < tile.rows; c += 64) {
                uint32_t v[32];
                const float as_lane = c + lane < tile.rows ? p.a_scale[tile.row0 + c + lane] : 0.0f;
                tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * ACC_COLS + c), v);
                tmem_ld_wait();
                Out *out = static_cast<Out *>(p.out) + (long long)(tile.row0 + c) * p.out_stride + ch;
                const int left = tile.rows - c;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float as = __shfl_sync(0xffffffffu, as_lane, j);
                    if (in && j < left) store_scaled(out, (int)v[j], as, bs);
                    out += p.out_stride;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (rank == 0) mbar_arrive(bar_tempty + 8 * acc);
                else mbar_arrive_cluster(lead_tempty + 8 * acc);
            }
            if ((acc ^= 1) == 0) acc_phase ^= 1u;
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();          // the peer no longer signals this CTA's barriers or reads its operands
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
        if (CTAS == 1) tmem_dealloc_self(tmem, 2 * ACC_COLS);
        else tmem_dealloc(tmem, 2 * ACC_COLS);
    }
}

// The operands as the tensor maps need them.  A map's box and the kernel's tile come from the same constant, in the two functions below.
struct QmOperands { const void *a, *b; long long b_rows, a_stride, b_stride; };

bool encode_operands(const QmP &p, const QmOperands &o, int token_rows, CUtensorMap *a, CUtensorMap *b)
{
    return encode_tiles(b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, o.b, p.k, o.b_rows, o.b_stride, 0, 0, QM_ROWS) &&
           encode_tiles(a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, o.a, p.k, p.rows, o.a_stride, 0, 0, token_rows);
}

template <int BN, int SPLITS, typename Out>
int launch_split(const QmP &p, const QmOperands &o, int device, cudaStream_t stream)
{
    CUtensorMap a, b;
    if (!encode_operands(p, o, BN, &a, &b)) return MOE_OVL_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    const auto kernel = quant_matmul_kernel<BN, SPLITS, Out>;
    if (!allow_smem(kernel, QmShape<BN>::SMEM, device, allowed)) return MOE_OVL_ERR_CUDA;
    // most token tiles that any counts can give
    const long long tiles = p.counts ? p.rows / BN + std::min(p.experts, p.rows) : (p.rows - 1) / BN + 1;
    const long long blocks = tiles * p.row_tiles * SPLITS;
    if (blocks > 0x7fffffffll) return MOE_OVL_ERR_UNSUPPORTED;
    return launch_behind(kernel, (unsigned)blocks, dim3(QM_THREADS), QmShape<BN>::SMEM, SPLITS, stream, b, a, p);
}

template <int CTAS, int TOKENS, typename Out>
int launch_tiles(const QmP &p, const QmOperands &o, int device, cudaStream_t stream)
{
    CUtensorMap a, b;
    if (!encode_operands(p, o, TOKENS / CTAS, &a, &b)) return MOE_OVL_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    const auto kernel = quant_matmul_tiles_kernel<CTAS, TOKENS, Out>;
    if (!allow_smem(kernel, QpShape<CTAS, TOKENS>::SMEM, device, allowed)) return MOE_OVL_ERR_CUDA;
    return launch_behind(kernel, (unsigned)(sm_count(device) / CTAS * CTAS), dim3(QP_THREADS), QpShape<CTAS, TOKENS>::SMEM, CTAS, stream, b, a, p);
}

template <int N> struct Number { static constexpr int value = N; };

// ctas 0: a cluster of `splits` CTAs per tile; 1, 2: persistent CTAs, alone or in pairs.
struct QmChoice { int ctas, tokens, splits; };

// The kernel goes by the tiles there are (with the experts' rows taken as even: the counts are on the device).  Measured, us:
//   few tiles leave SMs idle, so they share their K: 1 token, n = k = 4096 (32 tiles) 7.3 split by 4, 8.0 unsplit; n = 1024, k = 8192 5.4 split
//     by 8, 11.7; 128 tokens, n = 4096, k = 14336 (64 tiles) 18.1 and 20.9.  A step of K takes a CTA about 0.15 us; sharing costs about 1.2 us, and
//     0.03 us per token of the tile, whose parts have to be added up (0.3 us less since the scales are asked for early: 6.0, 5.0 and 16.8 now).  With more
//     tiles it does not pay: n = 8192, k = 2048 (64) 7.3 and 6.8;
//   up to 64 tokens per expert, or where tiles of 64 fit one wave of the 148 CTAs, single CTAs: 16 experts of 64 tokens 48.4 against 49.4 in
//     pairs (of 128: 61.1 against 55.8); 256 tokens, n = k = 4096 9.4 against 11.7.  Tiles of 32 where those fit the wave: 64 tokens, n = k = 4096
//     8.5 against 9.2;
//   experts' rows are never even, and a second tile reads an expert's weights anew, so their tiles are taken wider, where the mean is above 4
//     rows (64 experts of 15 rows, the busiest 65, n = 224, k = 3312: 17.6 with tiles of 16, 14.0 of 32, 14.8 of 64; 16 experts of 32, the busiest
//     158, n = 8192, k = 2048: 49.2 with 32, 45.8 with 64; one row each, n = 5104, k = 3088: 33.4 with 16, 35.7 with 32, 42.9 with 64);
//   pairs take 128 or 256 tokens, whose tiles cost about 8 : 13: 512 tokens, n = k = 4096 (one wave of the 74 pairs each) 12.2 and 17.2; 2048
//     tokens (four waves, two) 28.9 and 26.9.
QmChoice choose(const QmP &p)
{
    const int groups = p.experts ? std::min(p.experts, p.rows) : 1, per_group = (p.rows - 1) / groups + 1;
    auto tiles = [&](int channels, int tokens) {
        return (long long)((p.n - 1) / channels + 1) * groups * ((per_group - 1) / tokens + 1);
    };
    const long long ksteps = (p.k + QM_K - 1) / QM_K;
    QmChoice c = {0, per_group <= 16 ? 16 : per_group <= 64 ? 32 : 64, 1};
    const long long shared = tiles(QM_ROWS, c.tokens);
    if (shared <= (ksteps >= 64 ? 74 : 40)) {
        // two CTAs per SM at most, a step of K for each, eight of them only for a long K
        while (c.splits < 8 && shared * c.splits * 2 <= 296 && c.splits * 2 <= ksteps && (c.splits < 4 || ksteps >= 64)) c.splits *= 2;
        if (ksteps * (c.splits - 1) * 15 > c.splits * (120 + 3 * std::min(c.tokens, per_group))) return c;
    }
    if (p.experts && per_group > 4 && per_group <= 64) return {1, per_group <= 16 ? 32 : 64, 1};
    if (per_group <= 16) return {1, 16, 1};
    if (per_group <= 32 || tiles(QM_ROWS, 32) <= 148) return {1, 32, 1};
    if (per_group <= 64 || tiles(QM_ROWS, 64) <= 148) return {1, 64, 1};
    const long long w128 = (tiles(2 * QM_ROWS, 128) + 73) / 74, w256 = (tiles(2 * QM_ROWS, 256) + 73) / 74;
    return {2, per_group <= 128 || 8 * w128 <= 13 * w256 ? 128 : 256, 1};
}

}  // namespace

extern "C" int moe_ovl_quant_matmul(const moe_ovl_quant_matmul_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->n < 1 || a->k < 1 || a->num_experts < 0 ||
        (a->flags & ~MOE_OVL_QUANT_MATMUL_TEST_NO_LOADS) != 0 || a->wait_timeout_us < 0 ||
        !known_dtype(a->out_dtype) || (a->num_experts > 0) != (a->expert_counts != nullptr))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->k > MOE_OVL_MAX_QUANT_K || a->k % 16 != 0 || a->num_experts > 1024) return MOE_OVL_ERR_UNSUPPORTED;
    const long long b_rows = (long long)std::max(a->num_experts, 1) * a->n;
    if (b_rows > 0x7fffffffll) return MOE_OVL_ERR_UNSUPPORTED;
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->out_dtype);
    if (!a->a || !a->a_scale || !a->b || !a->b_scale || !a->out || !a->status || !aligned(a->a_scale, 4) || !aligned(a->b_scale, 4) ||
        !aligned(a->out, es) || !aligned(a->status, 4) || !aligned(a->expert_counts, 4) || (a->rows > 1 && (a->a_stride < a->k || a->out_stride < a->n)) ||
        (b_rows > 1 && a->b_stride < a->k))
        return MOE_OVL_ERR_INVALID_ARG;
    if (std::max(std::max(a->a_stride, a->b_stride), a->out_stride) > 0x7fffffff) return MOE_OVL_ERR_UNSUPPORTED;
    // a single row's stride is never used; the tensor map wants one that holds the row
    const long long sa = a->rows > 1 ? a->a_stride : a->k, sb = b_rows > 1 ? a->b_stride : a->k;
    if (!aligned(a->a, 16) || !aligned(a->b, 16) || sa % 16 != 0 || sb % 16 != 0) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const QmP p = {a->rows, a->n, a->k, a->num_experts, (a->n - 1) / QM_ROWS + 1, a->expert_counts, a->a_scale, a->b_scale, a->out,
                   a->out_stride, a->status, a->wait_timeout_us > 0 ? a->wait_timeout_us * 1000ull : TILE_TIMEOUT_NS,
                   (a->flags & MOE_OVL_QUANT_MATMUL_TEST_NO_LOADS) != 0};
    const QmChoice c = choose(p);
    const QmOperands o = {a->a, a->b, b_rows, sa, sb};
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    return with_dtype(a->out_dtype, [&](auto t) {
        using Out = decltype(t);
        if (c.ctas == 1) {
            switch (c.tokens) {
            case 16: return launch_tiles<1, 16, Out>(p, o, a->device, stream);
            case 32: return launch_tiles<1, 32, Out>(p, o, a->device, stream);
            default: return launch_tiles<1, 64, Out>(p, o, a->device, stream);
            }
        }
        if (c.ctas == 2) {
            switch (c.tokens) {
            case 128: return launch_tiles<2, 128, Out>(p, o, a->device, stream);
            default: return launch_tiles<2, 256, Out>(p, o, a->device, stream);
            }
        }
        auto split = [&](auto n) {
            constexpr int BN = decltype(n)::value;
            switch (c.splits) {
            case 2: return launch_split<BN, 2, Out>(p, o, a->device, stream);
            case 4: return launch_split<BN, 4, Out>(p, o, a->device, stream);
            default: return launch_split<BN, 8, Out>(p, o, a->device, stream);
            }
        };
        switch (c.tokens) {
        case 16: return split(Number<16>());
        case 32: return split(Number<32>());
        default: return split(Number<64>());
        }
    });
}
