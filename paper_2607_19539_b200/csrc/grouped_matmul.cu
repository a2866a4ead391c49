// Products of 16-bit floats grouped by expert, and their gradients (moe_ovl_grouped_matmul, moe_ovl_grouped_matmul_backward in include/moe_ovl.h):
//   out[m][n]   = sum_k a[m][k] * b[e][n][k], or a[m][k] * b[e][k][n]      (m a row of expert e)
//   dweight[e][n][k] = sum over the rows m of expert e of dy[m][n] * x[m][k]
//
// One kernel for the three.  The matrix instruction's M side is what lies next to each other in the output (n of out, k of dweight), 128 of them per CTA, one
// per lane of the accumulator, so that a warp's 32 lanes store 32 neighbours; its N side is the output's rows, of which there may be few
// (a decode batch's tokens) and whose number goes in steps of 16.  Operands are taken from where they lie: with K (what is summed over) along their rows, or
// down their columns, which the instruction's descriptors tell apart, so no matrix is transposed in memory.
// The gradient of the weights sums over an expert's rows, which end anywhere inside a step of 64 rows.  What follows them belongs to the next expert
// and has to count as 0 on both sides (0 * NaN is NaN), so each expert's operands are read through tensor maps of its own, cut off at its last
// row; a small kernel in front writes them into the workspace.
#include <algorithm>

#include "matmul_tiles.cuh"

using namespace moe_ovl;

namespace {

constexpr int GM_K = STAGE_ROW / 2;          // K per pipeline stage
constexpr int GM_BOX = STAGE_ROW * GM_K;     // bytes of 64 columns x 64 rows, K down the columns
constexpr int GM_M_BYTES = TILE_CHANNELS * STAGE_ROW;

// The tensor cores cut a sum off where they add to it, instead of rounding: its error grows with the number of steps, 8.4e-6 of a gradient over 6000 rows where 32-bit
// sums are off by 9e-7, and 1.4e-2 of 2^21 terms of one sign, many times the rounding of 16 bits.  So a sum ends after 512 of K for 32-bit outputs and after 4096 for 16-bit ones, and the finishing
// warps add the pieces up in registers; a gradient's sums have no other end, so that no wait for one is long.
constexpr int segment_of(bool wide) { return (wide ? 512 : 4096) / GM_K; }

// What K runs along: rows of both operands; columns of the M side's; columns of both
enum { FORM_ROWS = 0, FORM_MIXED = 1, FORM_COLUMNS = 2 };

struct GmP {
    int rows, n, k, experts;                 // n: the M side; k: sum, or (FORM_COLUMNS) the N side
    int row_tiles;                           // tiles of the M side
    const int *counts;
    void *out;
    long long out_stride, out_far;           // between rows, between experts (FORM_COLUMNS)
    int *status;
    unsigned long long timeout_ns;
    uint32_t types;                          // of the instruction descriptor
    bool no_loads;                           // test hook
    bool accumulate;
    const CUtensorMap *expert_maps;          // FORM_COLUMNS: [experts][2]
    const int *order;                        // FORM_COLUMNS: experts, those with most rows first
};

// Operands with K down the columns: 64 columns x 8 rows of K are one swizzle atom of 1024 bytes; atoms follow each other along K, then (GM_BOX bytes
// on) along the columns.
__device__ __forceinline__ uint64_t columns_desc(uint32_t saddr)
{
    return (umma_smem_desc(saddr) & ~((uint64_t)0x3fff << 16)) | ((uint64_t)(GM_BOX >> 4) << 16);
}

template <int CTAS, int TOKENS, int FORM, int SPLITS_, typename Out> struct GmWork {
    static constexpr int SPLITS = SPLITS_;
    static constexpr int SHARE = TOKENS / CTAS;                              // of the N side, per CTA
    static constexpr int COLS = TOKENS < 32 ? 32 : TOKENS;                   // of tensor memory
    static constexpr int SEGMENT = segment_of(sizeof(Out) == 4);
    // Wide tiles whose sum is one piece go out as they are read, 32 columns at a time (96 rows of 16 experts, 8192 x 2048: 80.3 us, through the sums' registers 80.9)
    static constexpr bool ONE_PIECE = FORM != FORM_COLUMNS && sizeof(Out) == 2 && TOKENS >= 128;
    static constexpr int RING_BYTES = (SPLITS == 1 ? 200 : TOKENS > 64 ? 128 : 72) * 1024;
    static constexpr int PER_SM = SPLITS > 1 && TOKENS <= 64 ? 2 : 1;        // blocks: a cluster finds its place where there is room for another one
    using Shape = TileShape<CTAS, GM_M_BYTES + SHARE * STAGE_ROW, RING_BYTES, 2, COLS, 8, SEGMENT>;
    using Schedule = TileSchedule<CTAS * TILE_CHANNELS, TOKENS>;
    using Tile = typename Schedule::Tile;                                    // FORM_COLUMNS: row0, rows are those of the output
    const GmP &p;
    const CUtensorMap *map_m, *map_n;
    int *tile_start, *row_start;
    float *part;                             // SPLITS > 1: [TOKENS][TILE_CHANNELS], where the operands were: a part is written when the last of them has been read
    Schedule sched;
    int rank = 0, split = 0;

    struct From { const CUtensorMap *m, *n; int m0, n0, k0, expert; };

    __device__ __forceinline__ void begin(int lane)
    {
        fill_schedule<TOKENS>(p, tile_start, row_start, count_of(p, lane), lane);
        if constexpr (FORM == FORM_COLUMNS) {
            __syncwarp();
            for (int e = lane; e < groups(); e += 32) tile_start[e] = p.order[e];       // a table that this form has no use for
        }
    }
    __device__ __forceinline__ int groups() const { return p.counts ? p.experts : 1; }
    // FORM_COLUMNS: every expert has the same tiles, which take as long as it has rows.  The longest come first, and the workers take them to and fro, the first worker
    // first and then the last one first: of 49152 rows dealt out unevenly over 8 experts the busiest of 74 workers has 6 % more than the mean then, in the experts' order and always from the
    // first worker on 13 %.
    __device__ __forceinline__ long long total() const
    {
        if constexpr (FORM == FORM_COLUMNS) {
            const int workers = gridDim.x / (CTAS * SPLITS);
            return ((long long)groups() * p.row_tiles * ((p.k - 1) / TOKENS + 1) + workers - 1) / workers * workers;
        } else {
            return sched.total(groups());
        }
    }
    __device__ __forceinline__ Tile at(long long t)
    {
        if constexpr (FORM == FORM_COLUMNS) {
            const int workers = gridDim.x / (CTAS * SPLITS), wide = (p.k - 1) / TOKENS + 1, per = p.row_tiles * wide;
            const long long round = t / workers;
            if (round & 1) t = (2 * round + 1) * workers - 1 - t;
            const int e = (int)(t / per), i = (int)(t - (long long)e * per), row0 = i % wide * TOKENS;
            if (e >= groups()) return {0, 0, 0, 0};                     // the last round is not full
            return {tile_start[e], i / wide * (CTAS * TILE_CHANNELS), row0, min(TOKENS, p.k - row0)};
        } else {
            return sched.at(t);
        }
    }
    __device__ __forceinline__ int all_steps(const Tile &t) const
    {
        if (FORM == FORM_COLUMNS && t.rows == 0) return 0;
        return (int)(((unsigned)(FORM == FORM_COLUMNS ? row_start[t.expert + 1] - row_start[t.expert] : p.k) + GM_K - 1) / GM_K);
    }
    __device__ __forceinline__ int step_of(int all, int i) const { return (int)((long long)all * i / SPLITS); }
    __device__ __forceinline__ int steps(const Tile &t) const
    {
        const int all = all_steps(t);
        return SPLITS == 1 ? all : step_of(all, split + 1) - step_of(all, split);
    }
    // Fewer rows than a full tile: a narrower instruction, whose halves the CTAs of a pair hold.
    __device__ __forceinline__ int width(const Tile &t) const { return (t.rows + 16 * CTAS - 1) / (16 * CTAS) * (16 * CTAS); }
    __device__ __forceinline__ From operands(const Tile &t, bool leader) const
    {
        From f = {map_m, map_n, uniform(t.channel0 + rank * TILE_CHANNELS), uniform((int)((unsigned)t.row0 + (unsigned)(rank * (width(t) / CTAS)))), 0, uniform(t.expert)};
        if constexpr (SPLITS > 1) f.k0 = uniform(step_of(all_steps(t), split) * GM_K);
        if constexpr (FORM == FORM_COLUMNS) {
            f.m = p.expert_maps + 2 * f.expert, f.n = f.m + 1;
            f.k0 += uniform(row_start[t.expert]);
            if (leader) {
                acquire_map(f.m);
                acquire_map(f.n);
            }
            if (SPLITS == 1 && p.accumulate) ask_for_output(t);
        }
        return f;
    }
    // What a tile is added to comes into L2 when its operands begin to come.
    __device__ __forceinline__ void ask_for_output(const Tile &t) const
    {
        constexpr int LINE = 128 / (int)sizeof(Out), LINES = TILE_CHANNELS / LINE;
        const int ch0 = t.channel0 + rank * TILE_CHANNELS;
        const Out *out = static_cast<const Out *>(p.out) + t.expert * p.out_far + (long long)t.row0 * p.out_stride;
        for (int i = threadIdx.x & 31; i < t.rows * LINES; i += 32) {
            const int ch = ch0 + i % LINES * LINE;
            if (ch < p.n) asm volatile("prefetch.global.L2 [%0];" ::"l"(out + (long long)(i / LINES) * p.out_stride + ch));
        }
        __syncwarp();
    }
    __device__ __forceinline__ static void acquire_map(const CUtensorMap *map)
    {
        asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(map) : "memory");
    }
    __device__ __forceinline__ void load(uint32_t on, const From &f, uint32_t sa, uint32_t bar, int step) const
    {
        const int k = f.k0 + step * GM_K;
        if constexpr (FORM == FORM_ROWS) {
            load_3d<CTAS>(on, sa, f.m, bar, k, f.m0, f.expert);
        } else if constexpr (FORM == FORM_MIXED) {
#pragma unroll
            for (int i = 0; i < TILE_CHANNELS / 64; ++i) load_3d<CTAS>(on, sa + i * GM_BOX, f.m, bar, f.m0 + 64 * i, k, f.expert);
        } else {
#pragma unroll
            for (int i = 0; i < TILE_CHANNELS / 64; ++i) load_2d<CTAS>(on, sa + i * GM_BOX, f.m, bar, f.m0 + 64 * i, k);
        }
        if constexpr (FORM == FORM_COLUMNS) {
#pragma unroll
            for (int i = 0; i < SHARE / 64; ++i) load_2d<CTAS>(on, sa + GM_M_BYTES + i * GM_BOX, f.n, bar, f.n0 + 64 * i, k);
        } else {
            load_2d<CTAS>(on, sa + GM_M_BYTES, f.n, bar, k, f.n0);
        }
    }
    __device__ __forceinline__ uint32_t instruction(const Tile &t) const
    {
        return p.types | (1u << 4) | (FORM != FORM_ROWS ? 1u << 15 : 0u) | (FORM == FORM_COLUMNS ? 1u << 16 : 0u) | ((uint32_t)(width(t) >> 3) << 17) |
               ((uint32_t)(CTAS * TILE_CHANNELS >> 4) << 24);
    }
    __device__ __forceinline__ void multiply(uint32_t on, uint32_t d, uint32_t stage16, uint32_t idesc, bool first, int) const
    {
        const uint64_t dm = (FORM == FORM_ROWS ? umma_smem_desc(0) : columns_desc(0)) + stage16;
        const uint64_t dn = (FORM == FORM_COLUMNS ? columns_desc(0) : umma_smem_desc(0)) + stage16 + GM_M_BYTES / 16;
        constexpr int STEP_M = FORM == FORM_ROWS ? 2 : 16 * STAGE_ROW / 16, STEP_N = FORM == FORM_COLUMNS ? 16 * STAGE_ROW / 16 : 2;
#pragma unroll
        for (int i = 0; i < GM_K / 16; ++i)
            umma_f16<CTAS>(on, d, dm + (uint64_t)(i * STEP_M), dn + (uint64_t)(i * STEP_N), idesc, first && i == 0 ? 0u : 1u);
    }
    __device__ __forceinline__ void close(int) const {}
    __device__ __forceinline__ void join(const Tile &t) const
    {
        Out *out = static_cast<Out *>(p.out) + (FORM == FORM_COLUMNS ? t.expert * p.out_far : 0) + (long long)t.row0 * p.out_stride;
        join_parts<SPLITS>(part, out, p.out_stride, t.channel0, p.n, t.rows, split, FORM == FORM_COLUMNS && p.accumulate);
    }
    // 32 rows of the output from row c of the tile on, one column per lane.
    __device__ __forceinline__ void store(const Tile &t, const float *sum, int c, int ch, bool in) const
    {
        if constexpr (SPLITS > 1) {
            float *own = part + c * TILE_CHANNELS + (ch - t.channel0);
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (c + j < TOKENS) own[j * TILE_CHANNELS] = sum[j];
            return;
        }
        Out *out = static_cast<Out *>(p.out) + (FORM == FORM_COLUMNS ? t.expert * p.out_far : 0) + (long long)(t.row0 + c) * p.out_stride + ch;
        const int left = in ? t.rows - c : 0;
        if (left >= 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j, out += p.out_stride) *out = from_f32<Out>(sum[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j, out += p.out_stride)
                if (j < left) *out = from_f32<Out>(sum[j]);
        }
    }
    __device__ __forceinline__ bool finish(const Tile &t, Accumulators<Shape> &accs, const GmP &, int warp, int lane) const
    {
        const int quarter = (warp + 2) & 3, half = warp >> 2;        // a warp reads the lanes of its position among four; every other 32 columns
        const int ch = t.channel0 + rank * TILE_CHANNELS + quarter * 32 + lane;
        const bool in = (unsigned)ch < (unsigned)p.n, none = steps(t) == 0;
        if (none && p.accumulate && SPLITS == 1) return true;
        if (ONE_PIECE && steps(t) <= SEGMENT) {
            if (!none && !accs.wait(p, t.row0)) return false;
            for (int c = half * 32; c < t.rows; c += 64) {
                uint32_t v[32] = {};
                if (!none) {
                    tmem_ld32(accs.columns() + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c, v);
                    tmem_ld_wait();
                }
                store(t, reinterpret_cast<const float *>(v), c, ch, in);
            }
            if (!none) accs.release();
            return true;
        }
        constexpr int MINE = TOKENS <= 32 ? 32 : TOKENS / 2;
        float acc[MINE] = {};
        if (half * 32 < COLS) {
            if (FORM == FORM_COLUMNS && SPLITS == 1 && p.accumulate) {
                // what is added to comes while the first segment is multiplied.  Lanes and rows outside the output read its last ones, so that no load waits behind a branch
                const Out *old = static_cast<const Out *>(p.out) + t.expert * p.out_far + (long long)t.row0 * p.out_stride + min(ch, p.n - 1);
#pragma unroll
                for (int c = 0; c < MINE; ++c) acc[c] = to_f32(old[(long long)min(half * 32 + c % 32 + c / 32 * 64, t.rows - 1) * p.out_stride]);
            }
            for (int k = 0; k < steps(t); k += SEGMENT) {
                if (!accs.wait(p, t.row0)) return false;
                const uint32_t from = accs.columns() + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 32);
#pragma unroll
                for (int c = 0; c < MINE; c += 8) {
                    uint32_t v[8];
                    tmem_ld8(from + c % 32 + c / 32 * 64, v);
                    tmem_ld_wait(v);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const float2 sum = add2(make_float2(acc[c + j], acc[c + j + 1]), make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])));
                        acc[c + j] = sum.x, acc[c + j + 1] = sum.y;
                    }
                }
                accs.release();
            }
#pragma unroll
            for (int c = 0; c < MINE; c += 32) store(t, &acc[c], half * 32 + c * 2, ch, in);
        } else {
            for (int k = 0; k < steps(t); k += SEGMENT) {
                if (!accs.wait(p, t.row0)) return false;
                accs.release();
            }
        }
        return true;
    }
};

// Bound by the tensor cores where there are many rows (49152 of 8 experts, 2816 x 2048: 347-377 us, 1.50-1.63 PFLOP/s, the tensor pipe at work for 96 % of the time; the gradient of those weights
// 382-414 us, 92 %), by the weights' way from HBM where there are few (96 rows of 16 experts, 8192 x 2048: 81 us, 6.7 TB/s).  Pairs of CTAs and tiles of 256 x 256 halve what a CTA needs out of L2
// for an operation; accumulators are double buffered, so that a tile is stored while the next one is multiplied.
template <int CTAS, int TOKENS, int FORM, int SPLITS, typename Out>
__global__ void __launch_bounds__(GmWork<CTAS, TOKENS, FORM, SPLITS, Out>::Shape::THREADS, GmWork<CTAS, TOKENS, FORM, SPLITS, Out>::PER_SM)
grouped_matmul_kernel(const __grid_constant__ CUtensorMap map_m, const __grid_constant__ CUtensorMap map_n, const __grid_constant__ GmP p)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ int s_tile_start[1025], s_row_start[1025];
    using Work = GmWork<CTAS, TOKENS, FORM, SPLITS, Out>;
    static_assert(SPLITS == 1 || TOKENS * TILE_CHANNELS * 4 <= Work::Shape::STAGES * Work::Shape::STAGE_BYTES, "room for the parts");
    float *part = reinterpret_cast<float *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    run_tiles(Work{p, &map_m, &map_n, s_tile_start, s_row_start, part, {s_tile_start, s_row_start, p.row_tiles}}, p, smem_raw);
}

// The tensor maps of one expert's rows: those of all rows, ending at its last one; and its place in the order of the tiles.  A warp per expert.
constexpr int MAPS_WARPS = 4;
__global__ void __launch_bounds__(32 * MAPS_WARPS)
expert_maps_kernel(const __grid_constant__ CUtensorMap map_m, const __grid_constant__ CUtensorMap map_n, const GmP p, CUtensorMap *maps, int *order)
{
    __shared__ __align__(128) CUtensorMap s_map[MAPS_WARPS][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e = blockIdx.x * MAPS_WARPS + warp;
    for (int i = lane; i < 64; i += 32)
        reinterpret_cast<uint32_t *>(s_map[warp])[i] = i < 32 ? reinterpret_cast<const uint32_t *>(&map_m)[i] : reinterpret_cast<const uint32_t *>(&map_n)[i - 32];
    after_previous();
    may_follow();
    const int experts = p.counts ? p.experts : 1;
    if (e >= experts) return;
    unsigned end = (unsigned)p.rows;
    int place = 0;
    if (p.counts) {
        // saturating at `rows`: sums of parts that are each at most that need 64 bits
        unsigned long long sum = 0;
        for (int i = lane; i <= e; i += 32) sum += (unsigned)min(max(p.counts[i], 0), p.rows);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        end = (unsigned)min(sum, (unsigned long long)p.rows);
        const int own = p.counts[e];
        for (int i = lane; i < experts; i += 32) place += p.counts[i] > own || (p.counts[i] == own && i < e) ? 1 : 0;
        place = __reduce_add_sync(0xffffffffu, place);
    }
    if (lane == 0) order[place] = e;
    __syncwarp();
    if (lane < 2) {
        // an expert in front of which there are no rows has none itself, and is never read; a map needs at least one
        const unsigned rows = max(end, 1u);
        asm volatile("tensormap.replace.tile.global_dim.shared::cta.b1024.b32 [%0], 1, %1;" ::"l"((unsigned long long)smem_u32(&s_map[warp][lane])), "r"(rows) : "memory");
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm volatile("tensormap.cp_fenceproxy.global.shared::cta.tensormap::generic.release.gpu.sync.aligned [%0], [%1], 128;"
                     ::"l"(maps + 2 * e + i), "r"(smem_u32(&s_map[warp][i])) : "memory");
}

struct GmMaps { CUtensorMap m, n; };

template <int CTAS, int TOKENS, int FORM, int SPLITS, typename Out>
int launch(const GmP &p, const GmMaps &maps, long long tiles, int device, cudaStream_t stream)
{
    using Work = GmWork<CTAS, TOKENS, FORM, SPLITS, Out>;
    constexpr int SMEM = Work::Shape::SMEM;
    static std::atomic<unsigned long long> allowed{0};
    const auto kernel = grouped_matmul_kernel<CTAS, TOKENS, FORM, SPLITS, Out>;
    if (!allow_smem(kernel, SMEM, device, allowed)) return MOE_OVL_ERR_CUDA;
    const unsigned blocks = SPLITS > 1 ? (unsigned)(tiles * SPLITS) : (unsigned)(sm_count(device) / CTAS * CTAS);
    return launch_behind(kernel, blocks, dim3(Work::Shape::THREADS), SMEM, CTAS * SPLITS, stream, maps.m, maps.n, p);
}
// Few tiles: `splits` (2, 4 or 8) CTAs for each.
template <int TOKENS, int FORM, typename Out>
int launch_split(int splits, const GmP &p, const GmMaps &maps, long long tiles, int device, cudaStream_t stream)
{
    switch (splits) {
    case 2: return launch<1, TOKENS, FORM, 2, Out>(p, maps, tiles, device, stream);
    case 4: return launch<1, TOKENS, FORM, 4, Out>(p, maps, tiles, device, stream);
    default: return launch<1, TOKENS, FORM, 8, Out>(p, maps, tiles, device, stream);
    }
}

// splits > 1: a cluster of that many CTAs per tile; tiles: the most that any counts can give.
struct GmChoice { int ctas, tokens, splits; long long tiles; };

// The kernel goes by the tiles there are (with the experts' rows taken as even: the counts are on the device).  Measured, us:
//   few tiles of up to 128 rows share their steps (splits_of); of 256 rows, n = k = 4096, that would be 15.6 against 14.0 in pairs;
//   up to 16 rows single CTAs, whose start is shorter: 1 row, n = 28672, k = 4096 39.7 against 43.3 in pairs of 128 rows, n = k = 128 2.8 and 3.3; and for more rows where
//     their tiles fit half of the SMs: 100 rows, n = k = 512 4.0 and 4.9.  Experts' rows are never even, so from a mean of 5 on they go in pairs: 80 rows of 16 experts, n = 8192, k = 2048
//     83.5 and 80.4, 96 of 64, n = 1408 45.1 and 43.3;
//   pairs take 128 or 256 rows, whose tiles cost about 8 : 13: 512 rows, n = k = 4096 (one wave of the 74 pairs each) 15.0 and 23.8, 2048 rows (four waves, two) 48.4 and 45.7; 4096 rows of 16
//     experts, n = 8192, k = 2048 149 and 129.
GmChoice choose(const GmP &p)
{
    const int groups = p.experts ? std::min(p.experts, p.rows) : 1, per_group = (p.rows - 1) / groups + 1;
    auto tiles = [&](int channels, int tokens) {
        return (long long)((p.n - 1) / channels + 1) * groups * ((per_group - 1) / tokens + 1);
    };
    if (per_group <= 128) {
        const int few = per_group <= 16 ? 16 : per_group <= 32 ? 32 : 64;
        const long long most = (long long)((p.n - 1) / TILE_CHANNELS + 1) * (p.counts ? p.rows / few + groups : (p.rows - 1) / few + 1);
        const int splits = splits_of(most, 2, (p.k - 1) / GM_K + 1, std::min(few, per_group), 150);
        if (splits > 1) return {1, few, splits, most};
        if ((per_group <= 16 && !(p.experts && per_group > 4)) || tiles(TILE_CHANNELS, 16) <= 74) return {1, 16, 1, 0};
        return {2, 128, 1, 0};
    }
    const long long w128 = (tiles(2 * TILE_CHANNELS, 128) + 73) / 74, w256 = (tiles(2 * TILE_CHANNELS, 256) + 73) / 74;
    return {2, 8 * w128 <= 13 * w256 ? 128 : 256, 1, 0};
}

uint32_t instruction_types(int dtype) { return dtype == MOE_OVL_BF16 ? (1u << 7) | (1u << 10) : 0u; }
CUtensorMapDataType map_type(int dtype) { return dtype == MOE_OVL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16; }
bool float16(int dtype) { return dtype == MOE_OVL_BF16 || dtype == MOE_OVL_F16; }
constexpr long long FAR = 1ll << 39;         // elements: the tensor map's limit on strides is 2^40 bytes

}  // namespace

extern "C" int moe_ovl_grouped_matmul(const moe_ovl_grouped_matmul_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->n < 1 || a->k < 1 || a->num_experts < 0 ||
        (a->transposed & ~1) != 0 || (a->flags & ~MOE_OVL_MATMUL_TEST_NO_LOADS) != 0 || a->wait_timeout_us < 0 || !float16(a->dtype) ||
        (a->out_dtype != a->dtype && a->out_dtype != MOE_OVL_F32) || (a->num_experts > 0) != (a->expert_counts != nullptr))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->num_experts > MOE_OVL_MAX_GROUPS || a->n > MOE_OVL_MAX_MATMUL || a->k > MOE_OVL_MAX_MATMUL) return MOE_OVL_ERR_UNSUPPORTED;
    if (a->rows == 0) return MOE_OVL_OK;
    const int experts = std::max(a->num_experts, 1), b_rows = a->transposed ? a->k : a->n, b_cols = a->transposed ? a->n : a->k;
    if (!a->a || !a->b || !a->out || !a->status || !aligned(a->out, dtype_bytes(a->out_dtype)) || !aligned(a->status, 4) || !aligned(a->expert_counts, 4) ||
        !aligned(a->a, 2) || !aligned(a->b, 2) || (a->rows > 1 && (a->a_stride < a->k || a->out_stride < a->n)) || (b_rows > 1 && a->b_stride < b_cols) ||
        (experts > 1 && a->b_expert_stride < 1))
        return MOE_OVL_ERR_INVALID_ARG;
    if (std::max(std::max(a->a_stride, a->b_stride), a->out_stride) > 0x7fffffff || a->b_expert_stride >= FAR) return MOE_OVL_ERR_UNSUPPORTED;
    // strides that are never used: the tensor map wants some that hold the row and are multiples of 16 bytes
    const long long sa = a->rows > 1 ? a->a_stride : (a->k + 7ll) / 8 * 8, sb = b_rows > 1 ? a->b_stride : (b_cols + 7ll) / 8 * 8;
    const long long far = experts > 1 ? a->b_expert_stride : sb;
    if (!aligned(a->a, 16) || !aligned(a->b, 16) || sa % 8 != 0 || sb % 8 != 0 || far % 8 != 0) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    GmP p = {};
    p.rows = a->rows, p.n = a->n, p.k = a->k, p.experts = a->num_experts, p.counts = a->expert_counts;
    p.out = a->out, p.out_stride = a->out_stride, p.status = a->status;
    p.timeout_ns = a->wait_timeout_us > 0 ? a->wait_timeout_us * 1000ull : TILE_TIMEOUT_NS;
    p.types = instruction_types(a->dtype), p.no_loads = (a->flags & MOE_OVL_MATMUL_TEST_NO_LOADS) != 0;
    const GmChoice c = choose(p);
    p.row_tiles = (p.n - 1) / (c.ctas * TILE_CHANNELS) + 1;
    GmMaps maps;
    const CUtensorMapDataType type = map_type(a->dtype);
    if (!encode_tiles(&maps.m, type, 2, a->b, b_cols, b_rows, 2 * sb, experts, 2 * far, a->transposed ? GM_K : TILE_CHANNELS) ||
        !encode_tiles(&maps.n, type, 2, a->a, a->k, a->rows, 2 * sa, 0, 0, c.tokens / c.ctas))
        return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    return with_dtype(a->out_dtype, [&](auto t) {
        using Out = decltype(t);
        auto form = [&](auto f) {
            constexpr int F = decltype(f)::value;
            if (c.splits > 1) {
                switch (c.tokens) {
                case 16: return launch_split<16, F, Out>(c.splits, p, maps, c.tiles, a->device, stream);
                case 32: return launch_split<32, F, Out>(c.splits, p, maps, c.tiles, a->device, stream);
                default: return launch_split<64, F, Out>(c.splits, p, maps, c.tiles, a->device, stream);
                }
            }
            if (c.ctas == 1) return launch<1, 16, F, 1, Out>(p, maps, 0, a->device, stream);
            return c.tokens == 128 ? launch<2, 128, F, 1, Out>(p, maps, 0, a->device, stream) : launch<2, 256, F, 1, Out>(p, maps, 0, a->device, stream);
        };
        return a->transposed ? form(std::integral_constant<int, FORM_MIXED>()) : form(std::integral_constant<int, FORM_ROWS>());
    });
}

extern "C" int moe_ovl_grouped_matmul_workspace_bytes(int32_t num_experts, size_t *bytes)
{
    if (!bytes || num_experts < 0) return MOE_OVL_ERR_INVALID_ARG;
    if (num_experts > MOE_OVL_MAX_GROUPS) return MOE_OVL_ERR_UNSUPPORTED;
    *bytes = (sizeof(CUtensorMap) * 2 + sizeof(int)) * (size_t)std::max(num_experts, 1);
    return MOE_OVL_OK;
}

extern "C" int moe_ovl_grouped_matmul_backward(const moe_ovl_grouped_matmul_backward_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->n < 1 || a->k < 1 || a->num_experts < 0 ||
        (a->accumulate & ~1) != 0 || (a->flags & ~MOE_OVL_MATMUL_TEST_NO_LOADS) != 0 || a->wait_timeout_us < 0 || !float16(a->dtype) ||
        (a->out_dtype != a->dtype && a->out_dtype != MOE_OVL_F32) || (a->num_experts > 0) != (a->expert_counts != nullptr))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->num_experts > MOE_OVL_MAX_GROUPS || a->n > MOE_OVL_MAX_MATMUL || a->k > MOE_OVL_MAX_MATMUL) return MOE_OVL_ERR_UNSUPPORTED;
    const int experts = std::max(a->num_experts, 1);
    size_t need = 0;
    moe_ovl_grouped_matmul_workspace_bytes(a->num_experts, &need);
    if (!a->dweight || !a->status || !aligned(a->dweight, dtype_bytes(a->out_dtype)) || !aligned(a->status, 4) || !aligned(a->expert_counts, 4) ||
        (a->rows > 0 && (!a->dy || !a->x || !aligned(a->dy, 2) || !aligned(a->x, 2))) || (a->rows > 1 && (a->dy_stride < a->n || a->x_stride < a->k)) ||
        (a->n > 1 && a->dweight_stride < a->k) || (experts > 1 && a->dweight_expert_stride < 1))
        return MOE_OVL_ERR_INVALID_ARG;
    if (!a->workspace || a->workspace_bytes < need || !aligned(a->workspace, 128)) return MOE_OVL_ERR_WORKSPACE;
    if (std::max(std::max(a->dy_stride, a->x_stride), a->dweight_stride) > 0x7fffffff || a->dweight_expert_stride >= FAR) return MOE_OVL_ERR_UNSUPPORTED;
    const long long sy = a->rows > 1 ? a->dy_stride : (a->n + 7ll) / 8 * 8, sx = a->rows > 1 ? a->x_stride : (a->k + 7ll) / 8 * 8;
    if (a->rows > 0 && (!aligned(a->dy, 16) || !aligned(a->x, 16) || sy % 8 != 0 || sx % 8 != 0)) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    // without rows the weights' gradient is still written: nothing is read, through maps of the workspace's own bytes
    const bool none = a->rows == 0;
    GmP p = {};
    p.rows = a->rows, p.n = a->k, p.k = a->n, p.experts = a->num_experts, p.counts = a->expert_counts;
    p.out = a->dweight, p.out_stride = a->dweight_stride, p.out_far = a->dweight_expert_stride, p.status = a->status;
    p.timeout_ns = a->wait_timeout_us > 0 ? a->wait_timeout_us * 1000ull : TILE_TIMEOUT_NS;
    p.types = instruction_types(a->dtype), p.no_loads = (a->flags & MOE_OVL_MATMUL_TEST_NO_LOADS) != 0, p.accumulate = a->accumulate != 0;
    CUtensorMap *expert_maps = static_cast<CUtensorMap *>(a->workspace);
    int *order = reinterpret_cast<int *>(expert_maps + 2 * experts);
    p.expert_maps = expert_maps, p.order = order;
    GmMaps maps;
    const CUtensorMapDataType type = map_type(a->dtype);
    if (!encode_tiles(&maps.m, type, 2, none ? a->workspace : a->x, a->k, std::max(a->rows, 1), 2 * sx, 0, 0, GM_K) ||
        !encode_tiles(&maps.n, type, 2, none ? a->workspace : a->dy, a->n, std::max(a->rows, 1), 2 * sy, 0, 0, GM_K))
        return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    const int rc = launch_behind(expert_maps_kernel, (unsigned)((experts + MAPS_WARPS - 1) / MAPS_WARPS), dim3(32 * MAPS_WARPS), 0, 1, stream, maps.m, maps.n, p, expert_maps, order);
    if (rc != MOE_OVL_OK) return rc;
    // Few tiles: 128 columns instead of 256, by one CTA each or by several that share the rows, or 64 columns by twice as many, two on an SM.  A step of 64 rows takes about 0.22, 0.31
    // and 0.43 us then.  Measured, us: 100000 rows, n = k = 512 286 unshared, 120 with four CTAs for 128 columns, 81 with eight for 64; 20000 rows, 1024 x 512 57, 27 and 35.
    const long long pairs = (long long)experts * ((p.n - 1) / 256 + 1) * ((p.k - 1) / 256 + 1);
    const bool pair = pairs > 37;
    p.row_tiles = (p.n - 1) / (pair ? 256 : 128) + 1;
    const long long tiles = (long long)experts * p.row_tiles * ((p.k - 1) / 128 + 1), narrow = (long long)experts * p.row_tiles * ((p.k - 1) / 64 + 1);
    const int steps = a->rows / experts / GM_K, splits = splits_of(tiles, 1, steps, 128, 150), narrow_splits = splits_of(narrow, 2, steps, 64, 150);
    const bool wide = (splits > 1 ? 31 : 22) * narrow_splits <= 43 * splits;
    return with_dtype(a->out_dtype, [&](auto t) {
        using Out = decltype(t);
        if (pair) return launch<2, 256, FORM_COLUMNS, 1, Out>(p, maps, 0, a->device, stream);
        if (!wide && narrow_splits > 1) return launch_split<64, FORM_COLUMNS, Out>(narrow_splits, p, maps, narrow, a->device, stream);
        if (splits > 1) return launch_split<128, FORM_COLUMNS, Out>(splits, p, maps, tiles, a->device, stream);
        return launch<1, 128, FORM_COLUMNS, 1, Out>(p, maps, 0, a->device, stream);
    });
}
