// Product of 8-bit integers with a scale per token and per channel, dense or per expert (moe_ovl_quant_matmul in
// include/moe_ovl.h):  out[m][n] = (sum_k a[m][k] * b[e][n][k]) * a_scale[m] * b_scale[e][n].
//
// The operands are swapped on the tensor cores: 128 weight rows (channels) are the matrix instruction's M side and
// BN tokens its N side, because the number of tokens is what varies (one, a handful, a ragged group) and N goes in steps
// of 16 while M does not.  The accumulator then has a channel per lane and a token per column: the channel's scale is one
// register, and a warp's 32 lanes store 32 neighbouring channels of a token.  Sums are exact 32-bit integers, so splitting
// K over the CTAs of a cluster and adding their parts changes nothing.
#include <algorithm>
#include <atomic>

#include "opcommon.cuh"
#include "ptx.cuh"

using namespace moe_ovl;

namespace {

constexpr int QM_ROWS = 128;                 // channels per CTA
constexpr int QM_K = 128;                    // K per pipeline stage: one 128-byte swizzle row
constexpr int QM_A_BYTES = QM_ROWS * QM_K;
constexpr int QM_THREADS = 192;              // load warp, MMA warp, 4 epilogue warps
constexpr unsigned long long QM_TIMEOUT_NS = 2000000000ull;

enum : long long { SITE_QM_EMPTY = 32, SITE_QM_FULL, SITE_QM_DONE };

struct QmP {
    int rows, n, k, experts;                 // experts 0: one matrix
    int row_tiles;                           // tiles of QM_ROWS channels per expert
    int splits;                              // CTAs of a cluster that share a tile's K
    const int *counts;
    const float *a_scale, *b_scale;
    void *out;
    long long out_stride;
    int *status;
    unsigned long long timeout_ns;
    bool no_loads;                           // test hook
};

struct QmTile { int expert, row0, rows; };   // rows 0: beyond the last tile

// The `index`-th tile of at most `height` tokens, experts in order.  One warp; every lane gets the answer.  Counts are
// cut so that no tile reaches beyond the rows there are.
__device__ QmTile find_tile(const QmP &p, int index, int height, int lane)
{
    if (!p.counts) {
        const long long row0 = (long long)index * height;
        if (row0 >= p.rows) return {0, 0, 0};
        return {0, (int)row0, min(height, p.rows - (int)row0)};
    }
    long long rows_before = 0;
    int tiles_before = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 32) {
        const int e = e0 + lane;
        long long upto = e < p.experts ? max(p.counts[e], 0) : 0;      // inclusive sums over the lanes
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const long long last = min(rows_before + upto, (long long)p.rows);
        long long first = __shfl_up_sync(0xffffffffu, last, 1);
        if (lane == 0) first = rows_before;
        const int mine = (int)(last - first), tiles = (mine + height - 1) / height;
        int tiles_upto = tiles;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, tiles_upto, o);
            if (lane >= o) tiles_upto += v;
        }
        const int start = tiles_before + tiles_upto - tiles;
        const unsigned hit = __ballot_sync(0xffffffffu, index >= start && index < start + tiles);
        if (hit) {
            const int owner = __ffs(hit) - 1;
            const int r = __shfl_sync(0xffffffffu, (int)first + (index - start) * height, owner);
            const int end = __shfl_sync(0xffffffffu, (int)last, owner);
            return {e0 + owner, r, min(height, end - r)};
        }
        tiles_before += __shfl_sync(0xffffffffu, tiles_upto, 31);
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

// A give-up leaves copies in flight: they have to land before the CTA's shared memory goes.  Bounded.
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity, unsigned long long limit_ns)
{
    const unsigned long long t0 = globaltimer_ns();
    while (!mbar_try_wait(bar, parity) && globaltimer_ns() - t0 < limit_ns) {}
}

// One tile (128 channels x BN tokens) per cluster; the cluster's CTAs share its K.
template <int BN, typename Out>
__global__ void __launch_bounds__(QM_THREADS)
quant_matmul_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, const QmP p)
{
    constexpr int STAGES = QmShape<BN>::STAGES, STAGE_BYTES = QmShape<BN>::STAGE_BYTES, TMEM_COLS = BN < 32 ? 32 : BN;
    extern __shared__ uint8_t smem_raw[];
    __shared__ QmTile s_tile;
    __shared__ uint32_t s_tmem;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar_full = smem_base + STAGES * STAGE_BYTES, bar_empty = bar_full + 8 * STAGES, bar_done = bar_empty + 8 * STAGES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % (unsigned)p.splits);
    const unsigned tile_index = blockIdx.x / (unsigned)p.splits;
    const int row_tile = (int)(tile_index % (unsigned)p.row_tiles);

    if (warp == 0) {
        const QmTile t = find_tile(p, (int)(tile_index / (unsigned)p.row_tiles), BN, lane);
        if (lane == 0) s_tile = t;
    } else if (warp == 1) {
        tmem_alloc_self(smem_u32(&s_tmem), TMEM_COLS);
    } else if (threadIdx.x == 64) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(bar_full + 8 * i, 1);
            mbar_init(bar_empty + 8 * i, 1);
        }
        mbar_init(bar_done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const QmTile tile = s_tile;
    const uint32_t tmem = s_tmem;
    const int steps_all = (p.k + QM_K - 1) / QM_K;
    const int k0 = steps_all * rank / p.splits, k1 = steps_all * (rank + 1) / p.splits;
    if (tile.rows > 0) {
        if (warp == 0 && lane == 0 && !p.no_loads) {
            const int y_b = tile.expert * p.n + row_tile * QM_ROWS;
            int stage = 0;
            uint32_t phase = 0;
            int issued = 0;
            for (int k = k0; k < k1; ++k, ++issued) {
                if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, p, SITE_QM_EMPTY, k)) break;
                const uint32_t sa = smem_base + stage * STAGE_BYTES;
                mbar_arrive_expect_tx(bar_full + 8 * stage, STAGE_BYTES);
                tma_load_2d_self(sa, &map_b, bar_full + 8 * stage, k * QM_K, y_b);
                tma_load_2d_self(sa + QM_A_BYTES, &map_a, bar_full + 8 * stage, k * QM_K, tile.row0);
                if (++stage == STAGES) stage = 0, phase ^= 1u;
            }
            if (issued < k1 - k0) {
                // gave up
                for (int i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i)
                    drain(bar_full + 8 * (i % STAGES), (uint32_t)(i / STAGES) & 1u, p.timeout_ns);
            }
        } else if (warp == 1 && lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            for (int k = k0; k < k1; ++k) {
                if (!mbar_wait(bar_full + 8 * stage, phase, p, SITE_QM_FULL, k)) break;
                tc_fence_after();
                const uint32_t sa = smem_base + stage * STAGE_BYTES;
                const uint64_t da = umma_smem_desc(sa), db = umma_smem_desc(sa + QM_A_BYTES);
#pragma unroll
                for (int i = 0; i < QM_K / 32; ++i)
                    umma_i8<1>(tmem, da + (uint64_t)(i * 2), db + (uint64_t)(i * 2), umma_idesc_i8(QM_ROWS, BN), (k > k0 || i > 0) ? 1u : 0u);
                umma_commit_one(bar_empty + 8 * stage);
                if (++stage == STAGES) stage = 0, phase ^= 1u;
            }
            umma_commit_one(bar_done);
        }
    }
    __syncwarp();
    if (tile.rows > 0) {
        // everybody waits: nothing of the pipeline is in use behind this point, and its memory can hold the parts
        mbar_wait(bar_done, 0, p, SITE_QM_DONE, tile.row0);
        __syncwarp();
        tc_fence_after();
    }
    if (tile.rows > 0 && warp >= 2) {
        const int quarter = warp & 3;                       // a warp reads the lanes of its position among four
        const int c = quarter * 32 + lane, ch = row_tile * QM_ROWS + c;
        if (p.splits == 1) {
            const float bs = ch < p.n ? p.b_scale[(long long)tile.expert * p.n + ch] : 0.0f;
            for (int t0 = 0; t0 < BN && t0 < tile.rows; t0 += 16) {
                uint32_t v[16];
                tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + t0, v);
                tmem_ld_wait();
                Out *out = static_cast<Out *>(p.out) + (long long)(tile.row0 + t0) * p.out_stride + ch;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (t0 + j < tile.rows && ch < p.n)
                        store_scaled(out + j * p.out_stride, (int)v[j], p.a_scale[tile.row0 + t0 + j], bs);
            }
        } else {
            for (int t0 = 0; t0 < BN && t0 < tile.rows; t0 += 16) {
                uint32_t v[16];
                tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + t0, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(smem_base + 4u * (uint32_t)((t0 + j) * QM_ROWS + c)), "r"(v[j]) : "memory");
            }
        }
    }
    if (p.splits > 1) {
        __syncwarp();
        cluster_sync_all();
        if (tile.rows > 0 && warp >= 2) {
            const int c = (warp - 2) * 32 + lane, ch = row_tile * QM_ROWS + c;
            const float bs = ch < p.n ? p.b_scale[(long long)tile.expert * p.n + ch] : 0.0f;
            for (int t = rank; t < tile.rows; t += p.splits) {
                int sum = 0;
                for (int s = 0; s < p.splits; ++s)
                    sum += (int)ld_shared_cluster_u32(map_to_cta(smem_base + 4u * (uint32_t)(t * QM_ROWS + c), (uint32_t)s));
                if (ch < p.n)
                    store_scaled(static_cast<Out *>(p.out) + (long long)(tile.row0 + t) * p.out_stride + ch, sum, p.a_scale[tile.row0 + t], bs);
            }
        }
        __syncwarp();
        cluster_sync_all();                                 // the parts stay until everybody has read them
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc_self(tmem, TMEM_COLS);
}

// ------------------------------------------------------------------ large products: CTA pairs

constexpr int QP_ROWS = 256;                 // channels per tile: 128 in each CTA of the pair
constexpr int QP_TOKENS = 256;               // tokens per tile: each CTA loads half of them
constexpr int QP_STAGE_BYTES = QM_A_BYTES + QP_TOKENS / 2 * QM_K;
constexpr int QP_STAGES = 6;
constexpr int QP_THREADS = 320;              // load warp, MMA warp, 8 epilogue warps
constexpr int QP_GROUP = 16;                 // token tiles that are worked on side by side, see QpSchedule
constexpr int QP_SMEM = QP_STAGES * QP_STAGE_BYTES + 1024 + 256;

// Order of the tiles: experts one after the other; inside an expert up to QP_GROUP token tiles form a group, and for each tile
// of channels all token tiles of the group come next to each other.  The CTA pairs that run side by side then share one
// tile of weights in L2, and the weights are read from HBM once per group (4096 tokens).  Every pair takes every
// gridDim/2-th tile, so a role only ever moves forward through the experts.
struct QpSchedule {
    const int *tile_start, *row_start;       // [experts + 1] token tiles and rows before each expert, in shared memory
    int row_tiles, expert = 0;
    struct Tile { int expert, channel0, row0, rows; };
    __device__ long long total(int experts) const { return (long long)tile_start[experts] * row_tiles; }
    __device__ Tile at(long long index)
    {
        while (index >= (long long)tile_start[expert + 1] * row_tiles) ++expert;
        const int tiles = tile_start[expert + 1] - tile_start[expert];
        const int i = (int)(index - (long long)tile_start[expert] * row_tiles);
        const int group = i / (QP_GROUP * row_tiles), first = group * QP_GROUP, wide = min(QP_GROUP, tiles - first);
        const int j = i - group * QP_GROUP * row_tiles;
        const int row0 = row_start[expert] + (first + j % wide) * QP_TOKENS;
        return {expert, j / wide * QP_ROWS, row0, min(QP_TOKENS, row_start[expert + 1] - row0)};
    }
};

// One warp fills the schedule's tables; counts are cut so that no tile reaches beyond the rows there are.
__device__ void fill_schedule(const QmP &p, int *tile_start, int *row_start, int lane)
{
    if (!p.counts) {
        if (lane == 0) {
            tile_start[0] = row_start[0] = 0;
            tile_start[1] = (p.rows + QP_TOKENS - 1) / QP_TOKENS;
            row_start[1] = p.rows;
        }
        return;
    }
    long long rows_before = 0;
    int tiles_before = 0;
    if (lane == 0) tile_start[0] = row_start[0] = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 32) {
        const int e = e0 + lane;
        long long upto = e < p.experts ? max(p.counts[e], 0) : 0;
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const long long last = min(rows_before + upto, (long long)p.rows);
        long long first = __shfl_up_sync(0xffffffffu, last, 1);
        if (lane == 0) first = rows_before;
        int tiles = ((int)(last - first) + QP_TOKENS - 1) / QP_TOKENS;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, tiles, o);
            if (lane >= o) tiles += v;
        }
        if (e < p.experts) {
            tile_start[e + 1] = tiles_before + tiles;
            row_start[e + 1] = (int)last;
        }
        tiles_before += __shfl_sync(0xffffffffu, tiles, 31);
        rows_before = __shfl_sync(0xffffffffu, last, 31);
    }
}

// Persistent, one CTA per SM, pairs of CTAs share every matrix instruction (cta_group::2): 256 channels x 256 tokens, each CTA
// holding its 128 channels and HALF of the tokens, which halves the operand bytes per SM against single CTAs -- at
// 8 bits the tensor cores eat operands as fast as at 16, and that traffic out of L2 is what bounds the other kernel on large products.
// Accumulators are double buffered (2 x 256 columns of tensor memory): a tile is scaled and stored while the next one runs.
template <typename Out>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(QP_THREADS, 1)
quant_matmul_pair_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, const QmP p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ int s_tile_start[1025], s_row_start[1025];
    __shared__ uint32_t s_tmem;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar_full = smem_base + QP_STAGES * QP_STAGE_BYTES, bar_empty = bar_full + 8 * QP_STAGES;
    const uint32_t bar_tfull = bar_empty + 8 * QP_STAGES, bar_tempty = bar_tfull + 16, bar_drain = bar_tempty + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const uint32_t lead_full = map_to_cta(bar_full, 0), lead_tempty = map_to_cta(bar_tempty, 0);

    if (warp == 0) {
        fill_schedule(p, s_tile_start, s_row_start, lane);
    } else if (warp == 1) {
        tmem_alloc(smem_u32(&s_tmem), 512);
    } else if (threadIdx.x == 64) {
        for (int i = 0; i < QP_STAGES; ++i) {
            mbar_init(bar_full + 8 * i, 1);           // the leader's load thread arrives, expecting both CTAs' bytes
            mbar_init(bar_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_tfull + 8 * i, 1);
            mbar_init(bar_tempty + 8 * i, 16);        // one arrival per epilogue warp of both CTAs
        }
        mbar_init(bar_drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    QpSchedule sched{s_tile_start, s_row_start, (p.n + QP_ROWS - 1) / QP_ROWS};
    const long long total = sched.total(p.experts > 0 ? p.experts : 1);
    const long long first = blockIdx.x >> 1, step = gridDim.x >> 1;
    const int ksteps = (p.k + QM_K - 1) / QM_K;

    if (warp == 0) {
        if (lane == 0 && !p.no_loads) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            long long issued = 0;
            for (long long t = first; ok && t < total; t += step) {
                const QpSchedule::Tile tile = sched.at(t);
                const int y_b = tile.expert * p.n + tile.channel0 + (int)rank * QM_ROWS;
                const int y_a = tile.row0 + (int)rank * ((tile.rows + 31) / 32 * 16);       // second half of the tile's tokens
                for (int k = 0; k < ksteps; ++k, ++issued) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, p, SITE_QM_EMPTY, t)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sa = smem_base + stage * QP_STAGE_BYTES, full = lead_full + 8 * stage;
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * stage, 2 * QP_STAGE_BYTES);
                    tma_load_2d(sa, &map_b, full, k * QM_K, y_b);
                    tma_load_2d(sa + QM_A_BYTES, &map_a, full, k * QM_K, y_a);
                    if (++stage == QP_STAGES) stage = 0, phase ^= 1u;
                }
            }
            if (!ok && rank == 0) {
                // gave up: wait for the copies of both CTAs (the peer stays until the cluster barrier at the end)
                for (long long i = issued > QP_STAGES ? issued - QP_STAGES : 0; i < issued; ++i)
                    drain(bar_full + 8 * (uint32_t)(i % QP_STAGES), (uint32_t)(i / QP_STAGES) & 1u, p.timeout_ns);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true;
            for (long long t = first; ok && t < total; t += step) {
                // fewer tokens than a full tile: a narrower instruction
                const uint32_t idesc = umma_idesc_i8(2 * QM_ROWS, (sched.at(t).rows + 31) / 32 * 32);
                ok = mbar_wait<true>(bar_tempty + 8 * acc, acc_phase ^ 1u, p, SITE_QM_DONE, t);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(acc * QP_TOKENS);
                for (int k = 0; k < ksteps; ++k) {
                    ok = mbar_wait(bar_full + 8 * stage, phase, p, SITE_QM_FULL, t);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_base + stage * QP_STAGE_BYTES;
                    const uint64_t da = umma_smem_desc(sa), db = umma_smem_desc(sa + QM_A_BYTES);
#pragma unroll
                    for (int i = 0; i < QM_K / 32; ++i)
                        umma_i8<2>(d, da + (uint64_t)(i * 2), db + (uint64_t)(i * 2), idesc, (k | i) != 0 ? 1u : 0u);
                    umma_commit_pair(bar_empty + 8 * stage);
                    if (++stage == QP_STAGES) stage = 0, phase ^= 1u;
                }
                if (!ok) break;
                umma_commit_pair(bar_tfull + 8 * acc);
                if ((acc ^= 1) == 0) acc_phase ^= 1u;
            }
            umma_commit_self(bar_drain);                // every MMA has finished before tensor memory goes
            drain(bar_drain, 0, p.timeout_ns);
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;          // lanes 32 * quarter .., every other 32 columns
        int acc = 0;
        uint32_t acc_phase = 0;
        for (long long t = first; t < total; t += step) {
            const QpSchedule::Tile tile = sched.at(t);
            const int ch = tile.channel0 + (int)rank * QM_ROWS + quarter * 32 + lane;
            const bool in = ch < p.n;
            const float bs = in ? p.b_scale[(long long)tile.expert * p.n + ch] : 0.0f;
            // a warp leaves the loop as one: what follows needs all of its lanes
            if (!__all_sync(0xffffffffu, mbar_wait(bar_tfull + 8 * acc, acc_phase, p, SITE_QM_DONE, t))) break;
            tc_fence_after();
            for (int c = half * 32; c < tile.rows; c += 64) {
                uint32_t v[32];
                const float as_lane = c + lane < tile.rows ? p.a_scale[tile.row0 + c + lane] : 0.0f;
                tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * QP_TOKENS + c), v);
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
    cluster_sync_all();          // the peer no longer signals this CTA's barriers or reads its operands
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, 512);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn()
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

// Rows of k bytes, `stride` bytes apart, in boxes of 128 bytes x box_rows rows with the 128-byte swizzle; what lies beyond the
// matrix is read as 0.
bool encode_bytes(CUtensorMap *map, const void *base, long long rows, int k, long long stride, int box_rows)
{
    const EncodeTiledFn f = encode_fn();
    if (!f) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)stride};
    const cuuint32_t box[2] = {QM_K, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
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

int sm_count(int device)
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

template <int BN, typename Out> int launch_split(const QmP &p, const CUtensorMap &b, const CUtensorMap &a, int device, cudaStream_t stream)
{
    constexpr int smem = QmShape<BN>::SMEM;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(quant_matmul_kernel<BN, Out>, smem, device, allowed)) return MOE_OVL_ERR_CUDA;
    // most token tiles that any counts can give
    const long long tiles = p.counts ? p.rows / BN + std::min(p.experts, p.rows) : (p.rows + BN - 1) / BN;
    const long long blocks = tiles * p.row_tiles * p.splits;
    if (blocks > 0x7fffffffll) return MOE_OVL_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(QM_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, quant_matmul_kernel<BN, Out>, b, a, p) == cudaSuccess ? MOE_OVL_OK : MOE_OVL_ERR_CUDA;
}

template <typename Out> int launch_pair(const QmP &p, const CUtensorMap &b, const CUtensorMap &a, int device, cudaStream_t stream)
{
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(quant_matmul_pair_kernel<Out>, QP_SMEM, device, allowed)) return MOE_OVL_ERR_CUDA;
    quant_matmul_pair_kernel<Out><<<sm_count(device) / 2 * 2, QP_THREADS, QP_SMEM, stream>>>(b, a, p);
    return launched();
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
        (b_rows > 1 && a->b_stride < a->k) || a->a_stride >= (1ll << 39) || a->b_stride >= (1ll << 39) || a->out_stride >= (1ll << 40))
        return MOE_OVL_ERR_INVALID_ARG;
    // a single row's stride is never used; the tensor map wants one that holds the row
    const long long sa = a->rows > 1 ? a->a_stride : a->k, sb = b_rows > 1 ? a->b_stride : a->k;
    if (!aligned(a->a, 16) || !aligned(a->b, 16) || sa % 16 != 0 || sb % 16 != 0) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    QmP p = {a->rows, a->n, a->k, a->num_experts, (a->n + QM_ROWS - 1) / QM_ROWS, 1, a->expert_counts, a->a_scale, a->b_scale,
             a->out, a->out_stride, a->status,
             a->wait_timeout_us > 0 ? a->wait_timeout_us * 1000ull : QM_TIMEOUT_NS, (a->flags & MOE_OVL_QUANT_MATMUL_TEST_NO_LOADS) != 0};
    const int per_group = a->num_experts ? (a->rows + a->num_experts - 1) / a->num_experts : a->rows;
    const int bn = per_group <= 16 ? 16 : per_group <= 32 ? 32 : per_group <= 64 ? 64 : 128;
    // K is shared where the tiles alone would leave SMs idle
    const long long tiles = (long long)p.row_tiles * ((per_group + bn - 1) / bn) * std::max(1, std::min(a->num_experts, a->rows));
    while (p.splits < 8 && tiles * p.splits * 2 <= 296 && p.splits * 2 <= (a->k + QM_K - 1) / QM_K) p.splits *= 2;
    const bool pair = per_group > 256;
    CUtensorMap map_b, map_a;
    if (!encode_bytes(&map_b, a->b, b_rows, a->k, sb, QM_ROWS) || !encode_bytes(&map_a, a->a, a->rows, a->k, sa, pair ? QP_TOKENS / 2 : bn)) return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    return with_dtype(a->out_dtype, [&](auto t) {
        using Out = decltype(t);
        if (pair) return launch_pair<Out>(p, map_b, map_a, a->device, stream);
        switch (bn) {
        case 16: return launch_split<16, Out>(p, map_b, map_a, a->device, stream);
        case 32: return launch_split<32, Out>(p, map_b, map_a, a->device, stream);
        case 64: return launch_split<64, Out>(p, map_b, map_a, a->device, stream);
        default: return launch_split<128, Out>(p, map_b, map_a, a->device, stream);
        }
    });
}
