// Product of 8-bit floats (e4m3) with a scale for each block of 128, dense or per expert (moe_ovl_block_matmul in include/moe_ovl.h):
//   out[m][n] = sum over the blocks B of K of a_scale[m][B] * b_scale[e][n / 128][B] * (sum over k in B of a[m][k] * b[e][n][k]).
//
// A block's sum comes out of the tensor cores in 32 bits; the scales differ from block to block, so each block's sums are
// multiplied and added up in registers: one fused operation per output and block, beside the tensor cores' 128.  A step of the pipeline is one block
// of K, and accumulators in tensor memory go round step by step, so that the next block multiplies while this one is added.
//
// Many rows (BlockRows): rows of a on the matrix instruction's M side, one per lane of the accumulator.  A thread then holds one row,
// and the columns it adds up lie in one block of channels: one factor per thread and step.
// Few rows (BlockFew): channels on the M side and the rows on the N side, whose size goes in steps of 16; the weights are streamed, and the factors,
// one per row, are dealt out through shared memory.
#include <algorithm>

#include "matmul_tiles.cuh"

using namespace moe_ovl;

namespace {

constexpr int BM_M_BYTES = TILE_CHANNELS * STAGE_ROW;

struct BmP {
    int rows, n, k, experts;
    int row_tiles;                           // tiles of channels per expert
    int blocks, channel_blocks;              // of 128, along K and along n
    const int *counts;
    const float *a_scale, *b_scale;
    void *out;
    long long out_stride;
    int *status;
    unsigned long long timeout_ns;
    bool no_loads;                           // test hook
    bool wide;                               // rows of the output begin on 16 bytes
};

__device__ __forceinline__ float2 pair_of(const uint32_t *v) { return make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])); }

// Instruction descriptor: 32-bit sums of e4m3, K along the rows of both operands.
__device__ __forceinline__ uint32_t idesc_e4m3(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }
// One step: 128 values of K.  `n16`: where the N side's operand begins in its stage, / 16.
template <int CTAS> __device__ __forceinline__ void multiply_step(uint32_t on, uint32_t d, uint32_t stage16, uint32_t n16, uint32_t idesc)
{
    const uint64_t dm = umma_smem_desc(0) + stage16, dn = dm + n16;
#pragma unroll
    for (int i = 0; i < STAGE_ROW / 32; ++i) umma_f8<CTAS>(on, d, dm + (uint64_t)(i * 2), dn + (uint64_t)(i * 2), idesc, i > 0 ? 1u : 0u);
}

// ------------------------------------------------------------------ many rows

template <int CTAS, int CHANNELS, int SPLITS_, typename Out> struct BlockRows {
    static constexpr int SPLITS = SPLITS_, PITCH = TILE_CHANNELS + 4, TOKENS = CTAS * TILE_CHANNELS, PARTS = CHANNELS / 128, SHARE = 128 / CTAS, COLS = 128 * PARTS / 2;     // SHARE: of a part's channels, per CTA
    using Shape = TileShape<CTAS, BM_M_BYTES + PARTS * SHARE * STAGE_ROW, 136 * 1024, 4, 128, 8, 1, PARTS>;
    static constexpr int STAGE_OUT = 2 * 32 * 128;        // per finishing warp
    using Schedule = TileSchedule<CHANNELS, TOKENS>;
    using Tile = typename Schedule::Tile;
    const BmP &p;
    const CUtensorMap *map_a, *map_b, *map_out;
    int *tile_start, *row_start;
    uint8_t *stage;                          // [finishing warps][STAGE_OUT]
    float *part;                             // SPLITS > 1: [TOKENS][PITCH], where the operands were: a part is written when the last of them has been read
    Schedule sched;
    int rank = 0, split = 0;

    struct From { int a0, b0, expert, k0; };
    __device__ __forceinline__ void begin(int lane) { fill_schedule<TOKENS>(p, tile_start, row_start, count_of(p, lane), lane); }
    __device__ __forceinline__ long long total() const { return sched.total(p.counts ? p.experts : 1); }
    __device__ __forceinline__ Tile at(long long t) { return sched.at(t); }
    __device__ __forceinline__ int step_of(int i) const { return p.blocks * i / SPLITS; }
    __device__ __forceinline__ int steps(const Tile &) const { return SPLITS == 1 ? p.blocks : step_of(split + 1) - step_of(split); }
    __device__ __forceinline__ From operands(const Tile &t, bool) const
    {
        return {uniform((int)((unsigned)t.row0 + (unsigned)(rank * TILE_CHANNELS))), uniform(t.channel0 + rank * SHARE), uniform(t.expert), SPLITS == 1 ? 0 : uniform(step_of(split))};
    }
    __device__ __forceinline__ void load(uint32_t on, const From &f, uint32_t sa, uint32_t bar, int step) const
    {
        const int k = (f.k0 + step) * STAGE_ROW;
        load_2d<CTAS>(on, sa, map_a, bar, k, f.a0);
#pragma unroll
        for (int i = 0; i < PARTS; ++i) load_3d<CTAS>(on, sa + BM_M_BYTES + i * SHARE * STAGE_ROW, map_b, bar, k, f.b0 + i * 128, f.expert);
    }
    __device__ __forceinline__ uint32_t instruction(const Tile &) const { return idesc_e4m3(TOKENS, 128); }
    __device__ __forceinline__ void multiply(uint32_t on, uint32_t d, uint32_t stage16, uint32_t idesc, bool, int part) const
    {
        multiply_step<CTAS>(on, d, stage16, (BM_M_BYTES + part * SHARE * STAGE_ROW) / 16, idesc);
    }
    __device__ __forceinline__ bool finish(const Tile &t, Accumulators<Shape> &accs, const BmP &, int warp, int lane) const
    {
        const int quarter = (warp + Shape::CONTROL) & 3, half = PARTS == 1 ? warp >> 2 : 0;  // a warp reads the lanes of its position among four, and its part's columns or half of them
        const int in_tile = rank * TILE_CHANNELS + quarter * 32 + lane;
        const bool mine = in_tile < t.rows;
        const int block = t.channel0 / 128 + accs.group, ch0 = block * 128 + half * COLS;
        const int k0 = SPLITS == 1 ? 0 : step_of(split), all = steps(t);
        const float *sa = p.a_scale + (long long)(t.row0 + (mine ? in_tile : 0)) * p.blocks + k0;
        const float *sb = p.b_scale + ((long long)t.expert * p.channel_blocks + min(block, p.channel_blocks - 1)) * p.blocks + k0;
        float2 acc[COLS / 2];
#pragma unroll
        for (int i = 0; i < COLS / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
        float a_next = sa[0], b_next = sb[0];
        for (int k = 0; k < all; ++k) {
            if (!accs.wait(p, t.row0)) return false;
            const uint32_t from = accs.columns() + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * COLS);
            const float2 s = both(a_next * b_next);
            if (k + 1 < all) a_next = sa[k + 1], b_next = sb[k + 1];
            // 16 columns at a time: the sums take 128 of the 168 registers, and two chunks or wider ones push other values out of them
#pragma unroll
            for (int c = 0; c < COLS; c += 16) {
                uint32_t v[16];
                tmem_ld16(from + c, v);
                tmem_ld_wait(v);
                if (c + 16 == COLS) {
                    accs.release();               // all of them are in registers
                    accs.look();
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[c / 2 + j] = fma2(pair_of(&v[2 * j]), s, acc[c / 2 + j]);
            }
        }
        if constexpr (SPLITS > 1) {
            float *own = part + in_tile * PITCH + half * COLS;
#pragma unroll
            for (int i = 0; i < COLS; i += 4) *reinterpret_cast<float4 *>(own + i) = make_float4(acc[i / 2].x, acc[i / 2].y, acc[i / 2 + 1].x, acc[i / 2 + 1].y);
            return true;
        }
        if (t.rows > rank * TILE_CHANNELS + quarter * 32) store(t, acc, rank * TILE_CHANNELS + quarter * 32, ch0, stage + warp * STAGE_OUT, lane);
        return true;
    }
    __device__ __forceinline__ void join(const Tile &t) const
    {
        join_parts<SPLITS, PITCH>(part, static_cast<Out *>(p.out) + (long long)t.row0 * p.out_stride, p.out_stride, t.channel0, p.n, t.rows, split, false);
    }
    // A warp's 32 rows of COLS sums, 128 bytes of each row at a time: they are laid down in shared memory as a tile copy wants them, which takes them away while the warp goes on
    // with its next tile (7919 x 28672 x 4096 757 -> 731 us against the warp's own stores).  Rows that end inside the 32 (the next expert's follow) and outputs that a tile copy does not take are stored
    // by the warp, neighbours by neighbouring lanes.  A thread's own row straight from its registers would be 32 lines of memory per store, which took as long as nine steps of K.
    __device__ __forceinline__ void store(const Tile &t, const float2 (&acc)[COLS / 2], int row0, int ch0, uint8_t *own, int lane) const
    {
        constexpr int VEC = 16 / (int)sizeof(Out), WIDE = 128 / (int)sizeof(Out);
        const int rows = min(t.rows - row0, 32);
#pragma unroll
        for (int c0 = 0; c0 < COLS; c0 += WIDE) {
            const int left = p.n - ch0 - c0;
            uint8_t *buffer = own + c0 / WIDE % 2 * (STAGE_OUT / 2);
            // of the two buffers' copies the older one is this buffer's; where a row is one piece there is one buffer
            if (lane == 0) {
                if (COLS > WIDE) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                Pack<Out, VEC> pack;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int c = c0 + i * VEC + j;
                    pack.v[j] = from_f32<Out>(c & 1 ? acc[c / 2].y : acc[c / 2].x);
                }
                *reinterpret_cast<uint4 *>(buffer + lane * 128 + (i ^ (lane & 7)) * 16) = *reinterpret_cast<const uint4 *>(&pack);
            }
            if (p.wide && rows == 32 && left >= WIDE) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0)
                    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map_out), "r"(ch0 + c0), "r"(t.row0 + row0), "r"(smem_u32(buffer))
                                 : "memory");
            } else {
                __syncwarp();
                Out *out = static_cast<Out *>(p.out) + (long long)(t.row0 + row0) * p.out_stride + ch0 + c0;
                for (int row = 0; row < rows; ++row)
#pragma unroll
                    for (int c = 0; c < WIDE; c += 32) {
                        const int col = c + lane;
                        const Out v = *reinterpret_cast<const Out *>(buffer + row * 128 + ((col / VEC ^ row) & 7) * 16 + col % VEC * (int)sizeof(Out));
                        if (col < left) out[(long long)row * p.out_stride + col] = v;
                    }
            }
            // a group for each buffer, empty or not
            if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            __syncwarp();
        }
    }
    __device__ __forceinline__ void close(int lane) const
    {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
};

// ------------------------------------------------------------------ few rows

template <int TOKENS_, int SPLITS_, typename Out> struct BlockFew {
    static constexpr int SPLITS = SPLITS_, TOKENS = TOKENS_, COLS = TOKENS < 32 ? 32 : TOKENS;
    // Two groups of four warps take the steps in turn: what a warp does for one (a wait, its factors, 16 or 32 columns) takes longer than the weights of a step take to come.
    static constexpr int RING_BYTES = (SPLITS > 1 ? 64 : 80) * 1024;
    // Blocks: where the tiles are no multiple of the SMs, those that have two work on both at once (1 row, 28672 x 4096 22.7 -> 20.6 us; 40 rows of 32 experts, 2048 x 1408 12.4 -> 10.7).
    static constexpr int PER_SM = 2;
    using Shape = TileShape<1, BM_M_BYTES + TOKENS * STAGE_ROW, RING_BYTES, 256 / COLS, COLS, 8, 1, 1, 2>;
    using Schedule = TileSchedule<TILE_CHANNELS, TOKENS>;
    using Tile = typename Schedule::Tile;
    const BmP &p;
    const CUtensorMap *map_a, *map_b;
    int *tile_start, *row_start;
    float *factors;                          // [8 warps][2][TOKENS]
    float *part;                             // [TOKENS][TILE_CHANNELS]: the second group's sums, and with SPLITS > 1 this CTA's
    Schedule sched;
    int rank = 0, split = 0, turn = 0;       // turn: the group whose step is next
    bool lost = false;                       // a wait gave up

    struct From { int a0, b0, expert, k0; };
    __device__ __forceinline__ void begin(int lane) { fill_schedule<TOKENS>(p, tile_start, row_start, count_of(p, lane), lane); }
    __device__ __forceinline__ long long total() const { return sched.total(p.counts ? p.experts : 1); }
    __device__ __forceinline__ Tile at(long long t) { return sched.at(t); }
    __device__ __forceinline__ int step_of(int i) const { return p.blocks * i / SPLITS; }
    __device__ __forceinline__ int steps(const Tile &) const { return SPLITS == 1 ? p.blocks : step_of(split + 1) - step_of(split); }
    __device__ __forceinline__ From operands(const Tile &t, bool) const { return {uniform(t.row0), uniform(t.channel0), uniform(t.expert), SPLITS == 1 ? 0 : uniform(step_of(split))}; }
    __device__ __forceinline__ void load(uint32_t on, const From &f, uint32_t sa, uint32_t bar, int step) const
    {
        load_3d<1>(on, sa, map_b, bar, (f.k0 + step) * STAGE_ROW, f.b0, f.expert);
        load_2d<1>(on, sa + BM_M_BYTES, map_a, bar, (f.k0 + step) * STAGE_ROW, f.a0);
    }
    __device__ __forceinline__ uint32_t instruction(const Tile &) const { return idesc_e4m3(TILE_CHANNELS, TOKENS); }
    __device__ __forceinline__ void multiply(uint32_t on, uint32_t d, uint32_t stage16, uint32_t idesc, bool, int) const { multiply_step<1>(on, d, stage16, BM_M_BYTES / 16, idesc); }

    // The groups meet at barriers that have no time limit: a warp whose wait gave up goes on without waiting for sums.
    static constexpr int THERE = 1, TAKEN = 2;       // named barriers
    __device__ __forceinline__ static void meet(int barrier, bool waits)
    {
        if (waits) asm volatile("bar.sync %0, 256;" ::"r"(barrier) : "memory");
        else asm volatile("bar.arrive %0, 256;" ::"r"(barrier) : "memory");
    }
    __device__ __forceinline__ bool finish(const Tile &t, Accumulators<Shape> &accs, const BmP &, int warp, int lane)
    {
        constexpr int PER_LANE = (TOKENS + 31) / 32;
        const int quarter = (warp + Shape::CONTROL) & 3, ch = t.channel0 + quarter * 32 + lane;
        const int from = SPLITS == 1 ? 0 : step_of(split), all = steps(t);
        float *own = factors + warp * 2 * TOKENS;
        const float *sa = p.a_scale + (long long)t.row0 * p.blocks + from;
        const float *sb = p.b_scale + ((long long)t.expert * p.channel_blocks + t.channel0 / 128) * p.blocks + from;
        float2 acc[TOKENS / 2];
#pragma unroll
        for (int i = 0; i < TOKENS / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
        float a_next[PER_LANE] = {}, b_next = 0.0f;
        auto ask = [&](int k) {
            if (k >= all) return;
#pragma unroll
            for (int i = 0; i < PER_LANE; ++i)
                if (i * 32 + lane < t.rows) a_next[i] = sa[(long long)(i * 32 + lane) * p.blocks + k];
            b_next = sb[k];
        };
        const int k0 = (accs.group + turn) & 1;          // its first step of this tile
        turn = (turn + all) & 1;
        ask(k0);
        for (int k = k0; k < all; k += 2) {
            float *s = own + (k & 2) / 2 * TOKENS;       // two, so that a lane still reading the step before is not overtaken
#pragma unroll
            for (int i = 0; i < PER_LANE; ++i)
                if (i * 32 + lane < TOKENS) s[i * 32 + lane] = a_next[i] * b_next;
            ask(k + 2);
            __syncwarp();
            if (lost || !accs.wait(p, t.row0)) {
                lost = true;
                continue;
            }
            const uint32_t columns = accs.columns() + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
            for (int c = 0; c < TOKENS; c += 16) {
                if (c < t.rows) {
                    uint32_t v[16];
                    tmem_ld16(columns + c, v);
                    tmem_ld_wait(v);
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(s + c + j);
                        acc[(c + j) / 2] = fma2(pair_of(&v[j]), make_float2(f.x, f.y), acc[(c + j) / 2]);
                        acc[(c + j) / 2 + 1] = fma2(pair_of(&v[j + 2]), make_float2(f.z, f.w), acc[(c + j) / 2 + 1]);
                    }
                }
            }
            accs.release();
        }
        float *mine = part + quarter * 32 + lane;
        if (accs.group == 1) {
#pragma unroll
            for (int j = 0; j < TOKENS; ++j)
                if (j < t.rows) mine[j * TILE_CHANNELS] = j & 1 ? acc[j / 2].y : acc[j / 2].x;
            meet(THERE, false);
            if (SPLITS == 1) meet(TAKEN, true);
            return true;
        }
        meet(THERE, true);
#pragma unroll
        for (int j = 0; j < TOKENS; ++j) {
            if (j < t.rows) {
                float &sum = j & 1 ? acc[j / 2].y : acc[j / 2].x;
                sum += mine[j * TILE_CHANNELS];
                if (SPLITS > 1) mine[j * TILE_CHANNELS] = sum;
            }
        }
        if constexpr (SPLITS == 1) {
            meet(TAKEN, false);
            if ((unsigned)ch < (unsigned)p.n) {
                Out *out = static_cast<Out *>(p.out) + (long long)t.row0 * p.out_stride + ch;
#pragma unroll
                for (int j = 0; j < TOKENS; ++j) {
                    if (j < t.rows) *out = from_f32<Out>(j & 1 ? acc[j / 2].y : acc[j / 2].x);
                    out += p.out_stride;
                }
            }
        }
        return true;
    }
    __device__ __forceinline__ void close(int) const {}
    __device__ __forceinline__ void join(const Tile &t) const
    {
        join_parts<SPLITS>(part, static_cast<Out *>(p.out) + (long long)t.row0 * p.out_stride, p.out_stride, t.channel0, p.n, t.rows, split, false);
    }
};

// Bound by the finishing warps' steps: about 700 clocks for a wait, 128 columns read and added, and giving them back, where the tensor cores need 512 (7919 x 28672 x 4096: 731-750 us, 2.5 PFLOP/s, the
// tensor pipe at work for 74 % of the time).  A pair's tile of 256 x 256 takes all tensor memory for two steps, as four accumulators of 128 columns, each with four warps that add it up; wider ones would be
// given back later, more warps have too few registers for their sums.
template <int CTAS, int CHANNELS, int SPLITS, typename Out>
__global__ void __launch_bounds__(BlockRows<CTAS, CHANNELS, SPLITS, Out>::Shape::THREADS, 1)
block_matmul_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out, const __grid_constant__ BmP p)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ int s_tile_start[1025], s_row_start[1025];
    using Work = BlockRows<CTAS, CHANNELS, SPLITS, Out>;
    static_assert(SPLITS == 1 || (CTAS == 1 && CHANNELS == TILE_CHANNELS && Work::TOKENS * Work::PITCH * 4 <= Work::Shape::STAGES * Work::Shape::STAGE_BYTES), "room for the parts");
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    float *part = reinterpret_cast<float *>(ring);
    run_tiles(Work{p, &map_a, &map_b, &map_out, s_tile_start, s_row_start, ring + Work::Shape::STAGES * Work::Shape::STAGE_BYTES, part, {s_tile_start, s_row_start, p.row_tiles}}, p, smem_raw);
}

// Bound by the weights' way from HBM (1 x 28672 x 4096: 20.5-21.5 us, 5.5-5.7 TB/s); with few tiles by their steps one after the other, which clusters share then (1 x 512 x 4096: 4.8 us, 9.1 unshared).
template <int TOKENS, int SPLITS, typename Out>
__global__ void __launch_bounds__(BlockFew<TOKENS, SPLITS, Out>::Shape::THREADS, BlockFew<TOKENS, SPLITS, Out>::PER_SM)
block_matmul_few_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ BmP p)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ int s_tile_start[1025], s_row_start[1025];
    using Work = BlockFew<TOKENS, SPLITS, Out>;
    __shared__ __align__(16) float s_factors[Work::Shape::FINISHERS * 2 * TOKENS];
    run_tiles(Work{p, &map_a, &map_b, s_tile_start, s_row_start, s_factors, reinterpret_cast<float *>(smem_raw + Work::Shape::SMEM), {s_tile_start, s_row_start, p.row_tiles}}, p, smem_raw);
}

struct BmOperands { const void *a, *b; long long a_stride, b_stride, b_far, out_bytes; };       // out_bytes: between rows of the output

bool encode_operands(const BmP &p, const BmOperands &o, int a_rows, int b_rows, CUtensorMap *a, CUtensorMap *b)
{
    return encode_tiles(a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, o.a, p.k, p.rows, o.a_stride, 0, 0, a_rows) &&
           encode_tiles(b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, o.b, p.k, p.n, o.b_stride, std::max(p.experts, 1), o.b_far, b_rows);
}

template <int CTAS, int CHANNELS, int SPLITS, typename Out>
int launch_rows(BmP p, const BmOperands &o, long long tiles, int device, cudaStream_t stream)
{
    using Work = BlockRows<CTAS, CHANNELS, SPLITS, Out>;
    using Shape = typename Work::Shape;
    constexpr int SMEM = Shape::SMEM + Shape::FINISHERS * Work::STAGE_OUT;
    CUtensorMap a, b, out;
    p.row_tiles = (p.n - 1) / CHANNELS + 1;
    if (!encode_operands(p, o, TILE_CHANNELS, 128 / CTAS, &a, &b)) return MOE_OVL_ERR_CUDA;
    const CUtensorMapDataType type = sizeof(Out) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;       // moved, not looked at
    if (!p.wide) out = a;                    // not used
    else if (!encode_tiles(&out, type, sizeof(Out), p.out, p.n, p.rows, o.out_bytes, 0, 0, 32)) return MOE_OVL_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    const auto kernel = block_matmul_kernel<CTAS, CHANNELS, SPLITS, Out>;
    if (!allow_smem(kernel, SMEM, device, allowed)) return MOE_OVL_ERR_CUDA;
    const unsigned blocks = SPLITS > 1 ? (unsigned)(tiles * SPLITS) : (unsigned)(sm_count(device) / CTAS * CTAS);
    return launch_behind(kernel, blocks, dim3(Shape::THREADS), SMEM, CTAS * SPLITS, stream, a, b, out, p);
}

template <int TOKENS, int SPLITS, typename Out>
int launch_few(BmP p, const BmOperands &o, long long tiles, int device, cudaStream_t stream)
{
    using Work = BlockFew<TOKENS, SPLITS, Out>;
    constexpr int SMEM = Work::Shape::SMEM + TOKENS * TILE_CHANNELS * 4;
    CUtensorMap a, b;
    p.row_tiles = (p.n - 1) / TILE_CHANNELS + 1;
    if (!encode_operands(p, o, TOKENS, TILE_CHANNELS, &a, &b)) return MOE_OVL_ERR_CUDA;
    static std::atomic<unsigned long long> allowed{0};
    const auto kernel = block_matmul_few_kernel<TOKENS, SPLITS, Out>;
    if (!allow_smem(kernel, SMEM, device, allowed)) return MOE_OVL_ERR_CUDA;
    const unsigned blocks = SPLITS > 1 ? (unsigned)(tiles * SPLITS) : (unsigned)sm_count(device) * Work::PER_SM;
    return launch_behind(kernel, blocks, dim3(Work::Shape::THREADS), SMEM, SPLITS, stream, a, b, p);
}
template <int TOKENS, typename Out>
int launch_few(int splits, const BmP &p, const BmOperands &o, long long tiles, int device, cudaStream_t stream)
{
    switch (splits) {
    case 1: return launch_few<TOKENS, 1, Out>(p, o, tiles, device, stream);
    case 2: return launch_few<TOKENS, 2, Out>(p, o, tiles, device, stream);
    case 4: return launch_few<TOKENS, 4, Out>(p, o, tiles, device, stream);
    default: return launch_few<TOKENS, 8, Out>(p, o, tiles, device, stream);
    }
}

// ctas 0: few rows, `tile` of them; else `tile` channels.  splits > 1: a cluster of that many CTAs per tile; tiles: the most that any counts can give.
struct BmChoice { int ctas, tile, splits; long long tiles; };

// The kernel goes by the tiles there are (with the experts' rows taken as even: the counts are on the device).  Measured, us:
//   up to 32 rows on the N side: 32 rows, n = k = 4096 15.7, and 17.7 with the rows on the M side; 64 rows 16.8 and 14.3.  Experts' rows are never even, so from a mean of 5 on their tiles are
//     taken twice as high: 256 rows of 16 experts, n = 8192, k = 2048 47.4 and 46.9;
//   single CTAs or pairs: a pair's step of 256 x 256 takes about 0.54 us, a single one's of 128 x 128 0.35.  1024 rows, n = k = 4096 (two waves of the 148, one of the 74) 23.0 and 17.7; 512 rows 13.6 and 17.0;
//     2048 rows of 16 experts, n = 8192, k = 2048 68 and 77, 4096 rows 113 and 97;
//   few tiles share their steps (splits_of): 32 rows, n = k = 4096 15.7 alone, 7.6 shared, 128 rows 14.8 and 9.3.
BmChoice choose(const BmP &p)
{
    const int groups = p.experts ? std::min(p.experts, p.rows) : 1, per_group = (p.rows - 1) / groups + 1;
    auto most = [&](int height) { return (long long)p.channel_blocks * (p.counts ? p.rows / height + groups : (p.rows - 1) / height + 1); };
    if (per_group <= 32) {
        const int few = per_group <= 16 ? 16 : 32, splits = splits_of(most(few), 2, p.blocks, std::min(few, per_group), 280);
        if (splits > 1) return {0, few, splits, most(few)};
        return {0, p.experts && per_group > 4 ? 32 : few, 1, 0};
    }
    const long long singles = (long long)p.channel_blocks * groups * ((per_group - 1) / 128 + 1), pairs = (long long)((p.n - 1) / 256 + 1) * groups * ((per_group - 1) / 256 + 1);
    if ((singles + 147) / 148 * 35 > (pairs + 73) / 74 * 54) return {2, 256, 1, 0};
    return {1, 128, splits_of(most(TILE_CHANNELS), 1, p.blocks, std::min(TILE_CHANNELS, per_group), 350), most(TILE_CHANNELS)};
}

}  // namespace

extern "C" int moe_ovl_block_matmul(const moe_ovl_block_matmul_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->n < 1 || a->k < 1 || a->num_experts < 0 ||
        (a->flags & ~MOE_OVL_MATMUL_TEST_NO_LOADS) != 0 || a->wait_timeout_us < 0 || !known_dtype(a->out_dtype) ||
        (a->num_experts > 0) != (a->expert_counts != nullptr))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->num_experts > MOE_OVL_MAX_GROUPS || a->n > MOE_OVL_MAX_MATMUL || a->k > MOE_OVL_MAX_MATMUL) return MOE_OVL_ERR_UNSUPPORTED;
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->out_dtype), experts = std::max(a->num_experts, 1);
    if (!a->a || !a->a_scale || !a->b || !a->b_scale || !a->out || !a->status || !aligned(a->a_scale, 4) || !aligned(a->b_scale, 4) ||
        !aligned(a->out, es) || !aligned(a->status, 4) || !aligned(a->expert_counts, 4) || (a->rows > 1 && (a->a_stride < a->k || a->out_stride < a->n)) ||
        (a->n > 1 && a->b_stride < a->k) || (experts > 1 && a->b_expert_stride < 1))
        return MOE_OVL_ERR_INVALID_ARG;
    if (std::max(std::max(a->a_stride, a->b_stride), a->out_stride) > 0x7fffffff || a->b_expert_stride >= 1ll << 40) return MOE_OVL_ERR_UNSUPPORTED;
    // strides that are never used: the tensor map wants some that hold the row and are multiples of 16 bytes
    const long long sa = a->rows > 1 ? a->a_stride : (a->k + 15ll) / 16 * 16, sb = a->n > 1 ? a->b_stride : (a->k + 15ll) / 16 * 16;
    const long long far = experts > 1 ? a->b_expert_stride : sb;
    if (!aligned(a->a, 16) || !aligned(a->b, 16) || sa % 16 != 0 || sb % 16 != 0 || far % 16 != 0) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    BmP p = {};
    p.rows = a->rows, p.n = a->n, p.k = a->k, p.experts = a->num_experts, p.counts = a->expert_counts;
    p.blocks = (a->k - 1) / 128 + 1, p.channel_blocks = (a->n - 1) / 128 + 1;
    p.a_scale = a->a_scale, p.b_scale = a->b_scale, p.out = a->out, p.out_stride = a->out_stride, p.status = a->status;
    p.timeout_ns = a->wait_timeout_us > 0 ? a->wait_timeout_us * 1000ull : TILE_TIMEOUT_NS;
    p.no_loads = (a->flags & MOE_OVL_MATMUL_TEST_NO_LOADS) != 0;
    p.wide = aligned(a->out, 16) && (a->rows == 1 || a->out_stride * es % 16 == 0);
    // a single row's stride is never used: one that holds the row
    const BmOperands o = {a->a, a->b, sa, sb, far, a->rows > 1 ? a->out_stride * es : ((long long)a->n * es + 15) / 16 * 16};
    const BmChoice c = choose(p);
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    return with_dtype(a->out_dtype, [&](auto t) {
        using Out = decltype(t);
        if (c.ctas == 2) return launch_rows<2, 256, 1, Out>(p, o, 0, a->device, stream);
        if (c.ctas == 1) {
            switch (c.splits) {
            case 1: return launch_rows<1, 128, 1, Out>(p, o, 0, a->device, stream);
            case 2: return launch_rows<1, 128, 2, Out>(p, o, c.tiles, a->device, stream);
            case 4: return launch_rows<1, 128, 4, Out>(p, o, c.tiles, a->device, stream);
            default: return launch_rows<1, 128, 8, Out>(p, o, c.tiles, a->device, stream);
            }
        }
        return c.tile == 16 ? launch_few<16, Out>(c.splits, p, o, c.tiles, a->device, stream) : launch_few<32, Out>(c.splits, p, o, c.tiles, a->device, stream);
    });
}
