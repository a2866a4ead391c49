// Row operators in front of and between the expert products: RMS norm of a sum with an optional 8-bit output, its
// gradient, and the gated activation with an 8-bit output (entry points in include/moe_ovl.h).
//
// All of them read each element once, need one reduction over the row, and write once: aligned rows of up to 16384 columns of 16 bits are bound by
// HBM.  A row is held in registers between the two (NV packs of VEC elements per thread), so nothing is read twice; wider rows
// (f32: beyond 8192 columns) are more than 512 threads' registers hold and spill (norm of 4000 x 24576, bf16: 275 us where the bytes take 105).  The row's
// threads are one block, or one warp where the row is short (several rows per block then, and no block barrier).  Blocks
// stay and take rows at a fixed distance, and what belongs to a column (weights, the weight gradient's sums) stays in registers.
// The next row's loads are under way while a row is reduced and written: into registers, and in the gradient's kernel, which has
// three matrices to read and sums to keep, into shared memory (struct Feed).
#include <algorithm>
#include <atomic>
#include <utility>

#include "opcommon.cuh"

using namespace moe_ovl;

namespace {

constexpr float QUANT_MAX = 127.0f;
constexpr float QUANT_TINY = 7.8886090522101181e-31f;      // 2^-100
constexpr int NORM_PARTIALS = 888;                          // most partial rows of the weight gradient: 148 SMs x 6

// Threads a block of a kernel with so many values per thread may have: the row lives in registers.
constexpr int max_threads(int values) { return values <= 8 ? 1024 : 512; }
constexpr int swiglu_threads(int values) { return values <= 16 ? 1024 : 512; }     // 14336 columns fit a block of 896 threads, a row in 64 registers each

// Sums and largest values over the threads of one row.  `buf`: values of the row's warps, that no thread of the block still reads.
// In the second step every warp adds up all warps' values.
__device__ __forceinline__ float sum_of_warps(float v, int lane)
{
    const int warps = blockDim.x >> 5;
    v = lane < warps ? v : 0.0f;
    for (int o = warps > 16 ? 16 : warps > 8 ? 8 : warps > 4 ? 4 : 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return __shfl_sync(0xffffffffu, v, 0);
}
__device__ __forceinline__ float row_sum(float v, float *buf)
{
    v = warp_sum(v);
    if (blockDim.x == 32) return v;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    return sum_of_warps(buf[threadIdx.x & 31], threadIdx.x & 31);
}
__device__ __forceinline__ float row_max(float v, float *buf)
{
    v = warp_max(v);
    if (blockDim.x == 32) return v;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_max(lane < (int)(blockDim.x >> 5) ? buf[lane] : 0.0f);
}
__device__ __forceinline__ void row_sum_max(float &s, float &m, float2 *buf)
{
    s = warp_sum(s);
    m = warp_max(m);
    if (blockDim.x == 32) return;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = make_float2(s, m);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    // the same sum as sum_of_warps', in straight code: fewer instructions (norm of 16384 x 4096 to 8 bits 76 -> 71 us), more registers (gradient
    // 36 -> 43 us)
    const float2 t = lane < (int)(blockDim.x >> 5) ? buf[lane] : make_float2(0.0f, 0.0f);
    s = warp_sum(t.x);
    m = warp_max(t.y);
}

// The scale of a row whose largest magnitude is `most`, and the factor that takes its values to 8 bits; a row of (almost) nothing gives zeros.
// most / 127 is rounded once: the remainder of a first quotient is exact and brings it to within 2^-22 of a unit in the last place, while no
// quotient of 24 bits by 127 is nearer than 1/254 of one to the middle between two floats (Brisebarre and Muller, division by a constant).
__device__ __forceinline__ float quant_scale(float most)
{
    const float first = most * (1.0f / QUANT_MAX), rest = fmaf(-first, QUANT_MAX, most);
    return most < QUANT_TINY ? 0.0f : most < INFINITY ? fmaf(rest, 1.0f / QUANT_MAX, first) : most;
}
__device__ __forceinline__ float quant_factor(float most) { return most < QUANT_TINY ? 0.0f : QUANT_MAX / most; }
// VEC values in 8 bits: v * factor to the nearest whole number, ties to even.  Adding 1.5 * 2^23 rounds to a whole number and leaves it,
// as two's complement, in the float's low byte (|v * factor| <= 127 (1 + 2^-22): nothing to clamp); the conversion instruction has a
// fraction of that rate.  A row that holds a NaN or an infinity gives zeros: `keep` is 0 then.
// ROUNDED: the product is rounded as a value of its own first.  Values of few digits, as products of 16-bit ones are, often lie half-way
// between two steps, and the rounding takes most of these back to the half that the factor's error took them off (of 67 million values 470
// are a step off, fused 1200, of 32-bit torch operations 800).  The assembler makes one fused operation of a packed product and the sum behind it,
// but may not of a sum with +0.  Values that err by more than that already (the activation's) have no use for it.
template <bool ROUNDED> __device__ __forceinline__ float2 whole2(float2 v, float factor)
{
    const float2 magic = both(12582912.0f);
    if constexpr (ROUNDED) return add2(fma2(v, both(factor), both(0.0f)), magic);
    else return fma2(v, both(factor), magic);
}
template <int VEC, bool ROUNDED> __device__ __forceinline__ void store_quant(int8_t *q, const float *v, float factor, uint32_t keep)
{
    if constexpr (VEC == 1) {
        const float t = ROUNDED ? __fadd_rn(__fmul_rn(v[0], factor), 12582912.0f) : fmaf(v[0], factor, 12582912.0f);
        *q = (int8_t)(__float_as_uint(t) & keep);
    } else if constexpr (VEC == 2) {
        const float2 t = whole2<ROUNDED>(make_float2(v[0], v[1]), factor);
        *reinterpret_cast<uint16_t *>(q) = (uint16_t)(__byte_perm(__float_as_uint(t.x), __float_as_uint(t.y), 0x0040) & keep);
    } else {
        uint32_t b[VEC], w[VEC / 4];
#pragma unroll
        for (int j = 0; j < VEC; j += 2) {
            const float2 t = whole2<ROUNDED>(make_float2(v[j], v[j + 1]), factor);
            b[j] = __float_as_uint(t.x), b[j + 1] = __float_as_uint(t.y);
        }
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j)
            w[j] = __byte_perm(__byte_perm(b[4 * j], b[4 * j + 1], 0x0040), __byte_perm(b[4 * j + 2], b[4 * j + 3], 0x0040), 0x5410) & keep;
        if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(q) = w[0];
    }
}
__device__ __forceinline__ uint32_t keep_mask(float most) { return most <= 3.402823466e+38f ? 0xffffffffu : 0u; }

// Where row `row` of a matrix begins for a thread whose first column is c.  Rows are counted without sign: one step behind the last of 2^31 - 1
// rows is still a row number, but not one of a row that is read.  (The product of two signed numbers takes fewer registers.)
template <typename T> __device__ __forceinline__ T *at_row(T *base, unsigned row, int stride, int c) { return base + ((long long)(int)row * stride + c); }

// RAGGED rows: their length or their distance is no multiple of a pack, so they begin anywhere in one.  A thread then owns packs of the
// ADDRESS space: its first column is `shift` columns further left, and shift = (row * stride) mod VEC stays the same for a block when its
// rows lie a multiple of VEC rows apart.  All matrices have to agree on it (the same stride mod VEC, aligned bases).  Only the row's first and
// last pack are partial; their elements are read and written one by one, and count as 0 outside the row.  (4097 columns, 8000 rows, bf16:
// element by element 142 us, this way 75 us.)
template <int VEC, bool RAGGED> __device__ __forceinline__ bool whole_pack(int c, int d) { return RAGGED ? c >= 0 && c + VEC <= d : c < d; }
template <typename T, int VEC> __device__ __forceinline__ Pack<T, VEC> load_part(const T *p, int c, int d)
{
    Pack<T, VEC> r;
#pragma unroll
    for (int j = 0; j < VEC; ++j) r.v[j] = c + j >= 0 && c + j < d ? p[j] : from_f32<T>(0.0f);
    return r;
}
template <typename T, int VEC, bool RAGGED> __device__ __forceinline__ Pack<T, VEC> load_some(const T *p, int c, int d)
{
    if constexpr (RAGGED) {
        if (!whole_pack<VEC, true>(c, d)) return load_part<T, VEC>(p, c, d);
    }
    return load_pack<T, VEC>(p);
}
template <typename T, int VEC, bool RAGGED> __device__ __forceinline__ void store_some(T *p, const Pack<T, VEC> &r, int c, int d)
{
    if constexpr (RAGGED) {
        if (!whole_pack<VEC, true>(c, d)) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (c + j >= 0 && c + j < d) p[j] = r.v[j];
            return;
        }
    }
    store_pack<T, VEC>(p, r);
}
// The weights of a thread's columns, wherever they begin.
template <typename W, int VEC, bool RAGGED> __device__ __forceinline__ Pack<W, VEC> load_weight(const W *w, int c, int d)
{
    if constexpr (RAGGED) return load_part<W, VEC>(w + c, c, d);
    else return load_pack<W, VEC>(w + c);
}
template <int VEC, bool RAGGED> __device__ __forceinline__ void quant_some(int8_t *q, const float *v, float factor, uint32_t keep, int c, int d)
{
    if constexpr (RAGGED) {
        if (!whole_pack<VEC, true>(c, d)) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (c + j >= 0 && c + j < d) store_quant<1, true>(q + j, v + j, factor, keep);
            return;
        }
    }
    store_quant<VEC, true>(q, v, factor, keep);
}
template <int VEC, bool RAGGED> __device__ __forceinline__ int shift_of(unsigned row, int stride) { return RAGGED ? (int)(row * (unsigned)stride % VEC) : 0; }

// Two rows in shared memory, one in use and one on its way from global memory.  Every thread copies, waits for and reads its own
// packs only (asynchronous copies of 16 or 4 bytes), so no thread waits for another.  Partial packs are not copied.
template <typename T, int VEC, int NV, int ARRAYS, bool RAGGED> struct Feed {
    static constexpr int BYTES = VEC * (int)sizeof(T);
    uint32_t base, stride;                      // this thread's first pack, bytes from pack to pack
    int slot = 0;
    __device__ Feed()
    {
        extern __shared__ __align__(16) uint8_t feed_memory[];
        base = (uint32_t)__cvta_generic_to_shared(feed_memory) + (threadIdx.y * blockDim.x + threadIdx.x) * BYTES;
        stride = blockDim.x * blockDim.y * BYTES;
    }
    // Asks for a row into the slot that is not in use: `at[k]` where this thread's first column c lies in matrix k (NULL: none),
    // `across` columns from pack to pack.
    __device__ __forceinline__ void ask(const T *const (&at)[ARRAYS], bool any, int c, int d, int across)
    {
        if (any) {
#pragma unroll
            for (int k = 0; k < ARRAYS; ++k)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (at[k] && whole_pack<VEC, RAGGED>(c + i * across, d)) {
                        const uint32_t to = base + (((slot ^ 1) * ARRAYS + k) * NV + i) * stride;
                        if constexpr (BYTES == 16)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(at[k] + i * across) : "memory");
                        else
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(at[k] + i * across) : "memory");
                    }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ void turn() { slot ^= 1; }
    // The row of the slot in use is here; the one asked for last may not be.
    __device__ __forceinline__ void wait() const { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
    __device__ __forceinline__ Pack<T, VEC> got(int k, int i) const
    {
        Pack<T, VEC> r;
        const uint32_t from = base + ((slot * ARRAYS + k) * NV + i) * stride;
        if constexpr (BYTES == 16) {
            uint4 v;
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
            *reinterpret_cast<uint4 *>(&r) = v;
        } else {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
            *reinterpret_cast<uint32_t *>(&r) = v;
        }
        return r;
    }
};

struct NormP {
    unsigned rows;
    int d;
    float per_d, eps;                           // per_d: 1 / d
    const void *x, *residual, *weight;
    void *residual_out, *y;
    int8_t *q;
    float *scale, *rstd;
    int x_stride, residual_stride, residual_out_stride, y_stride, q_stride;
};

// The row's sum of squares and the largest |h * weight| come out of ONE reduction: rstd is a positive factor of the whole row,
// so the scale of the 8-bit output needs no second pass over the normed values.
template <typename T, typename W, int VEC, int NV, bool RAGGED>
__device__ __forceinline__ void add_norm_rows(const NormP &p)
{
    __shared__ float2 buf[2][32];
    after_previous();
    may_follow();
    const unsigned step = gridDim.x * blockDim.y;
    const W *w = static_cast<const W *>(p.weight);
    unsigned row = blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.rows) return;                  // whole warps: rows share a block only as one warp each
    const int c0 = threadIdx.x * VEC - shift_of<VEC, RAGGED>(row, p.x_stride), across = blockDim.x * VEC;
    Pack<T, VEC> a[NV], b[NV];
    auto load = [&](unsigned r) {
        const T *x = at_row(static_cast<const T *>(p.x), r, p.x_stride, c0), *res = at_row(static_cast<const T *>(p.residual), r, p.residual_stride, c0);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (c0 + i * across < p.d) {
                a[i] = load_some<T, VEC, RAGGED>(x + i * across, c0 + i * across, p.d);
                if (p.residual) b[i] = load_some<T, VEC, RAGGED>(res + i * across, c0 + i * across, p.d);
            }
    };
    load(row);
    Pack<W, VEC> wv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (c0 + i * across < p.d) wv[i] = load_weight<W, VEC, RAGGED>(w, c0 + i * across, p.d);
    for (int turn = 0; row < p.rows; row += step, turn ^= 1) {
        float v[NV * VEC];                      // h * weight
        float most = 0.0f;
        float2 sum = both(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (c0 + i * across >= p.d) continue;
            // the sum is rounded to the type it is stored in: the norm is that of the stored value
            if constexpr (VEC == 1) {
                if (p.residual) a[i].v[0] = from_f32<T>(to_f32(a[i].v[0]) + to_f32(b[i].v[0]));
                const float h = to_f32(a[i].v[0]);
                sum.x = fmaf(h, h, sum.x);
                v[i] = h * to_f32(wv[i].v[0]);
                most = max_abs(most, v[i]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    if (p.residual) add_round2(&a[i].v[j], &b[i].v[j]);
                    const float2 h = to_f32x2(&a[i].v[j]);
                    sum = fma2(h, h, sum);
                    const float2 t = mul2(h, to_f32x2(&wv[i].v[j]));
                    v[i * VEC + j] = t.x, v[i * VEC + j + 1] = t.y;
                    most = max_abs(most, t);
                }
            }
            if (p.residual_out)
                store_some<T, VEC, RAGGED>(at_row(static_cast<T *>(p.residual_out), row, p.residual_out_stride, c0) + i * across, a[i], c0 + i * across, p.d);
        }
        if (row + step < p.rows) load(row + step);
        float total = sum.x + sum.y;
        row_sum_max(total, most, buf[turn]);
        const float rstd = rsqrtf(fmaf(total, p.per_d, p.eps));
        if (threadIdx.x == 0 && p.rstd) p.rstd[row] = rstd;
        if (p.y) {
            T *y = at_row(static_cast<T *>(p.y), row, p.y_stride, c0);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (c0 + i * across < p.d) {
                    Pack<T, VEC> o;
                    if constexpr (VEC == 1) {
                        o.v[0] = from_f32<T>(v[i] * rstd);
                    } else {
#pragma unroll
                        for (int j = 0; j < VEC; j += 2)
                            from_f32x2(&o.v[j], mul2(make_float2(v[i * VEC + j], v[i * VEC + j + 1]), both(rstd)));
                    }
                    store_some<T, VEC, RAGGED>(y + i * across, o, c0 + i * across, p.d);
                }
            }
        }
        if (p.q) {
            int8_t *q = at_row(p.q, row, p.q_stride, c0);
            // rstd cancels out of a value over the row's largest
            const float value = most * rstd;
            if (threadIdx.x == 0) p.scale[row] = quant_scale(value);
            const float factor = value < QUANT_TINY ? 0.0f : QUANT_MAX / most;
            const uint32_t keep = keep_mask(value);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (c0 + i * across < p.d) quant_some<VEC, RAGGED>(q + i * across, v + i * VEC, factor, keep, c0 + i * across, p.d);
        }
    }
}

template <typename T, typename W, int VEC, int NV, bool RAGGED>
__global__ void __launch_bounds__(max_threads(VEC *NV)) add_norm_kernel(const NormP p) { add_norm_rows<T, W, VEC, NV, RAGGED>(p); }
// The same in fewer registers.
template <typename T, typename W, int VEC, int NV, bool RAGGED>
__global__ void __maxnreg__(VEC *NV <= 8 ? 40 : 128) add_norm_lean_kernel(const NormP p) { add_norm_rows<T, W, VEC, NV, RAGGED>(p); }

struct NormBackP {
    unsigned rows;
    int d;
    float per_d;
    const void *dy, *h, *weight, *d_residual;
    const float *rstd;
    void *dx;
    float *partial;                             // [gridDim.x][d] sums of dy * n, or NULL
    int dy_stride, h_stride, d_residual_stride, dx_stride;
};

// What the gradient's kernel asks of shared memory per row, where it takes rows through it: not for elements of two bytes, which the
// copies do not know, nor for rows of which no two fit.
template <typename T, int VEC, int NV> struct BackFeed {
    static constexpr int THREAD_BYTES = 3 * NV * VEC * (int)sizeof(T);
    static constexpr bool ON = VEC * sizeof(T) >= 4 && 2 * THREAD_BYTES * max_threads(VEC * NV) <= 200 * 1024;
};

// Every block (or warp) keeps its columns' share of the weight gradient over all of its rows; the partial rows are
// added up in a fixed order by reduce_partials_kernel: no atomics, the same bits every time.  A row is read from shared memory twice, before
// and after its reduction, so that few registers are in use across the barrier: blocks per SM carry this kernel (12289 x 2048,
// bf16: 84, 49, 40, 36 us with 1, 2, 3, 4 of them), not how many rows are on their way (one to four: the same).
template <typename T, typename W, int VEC, int NV, bool RAGGED>
__device__ __forceinline__ void add_norm_backward_rows(const NormBackP &p)
{
    constexpr bool FED = BackFeed<T, VEC, NV>::ON;
    __shared__ float buf[2][32];
    after_previous();
    may_follow();
    float acc[NV * VEC];
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i) acc[i] = 0.0f;
    const unsigned first = blockIdx.x * blockDim.y + threadIdx.y, step = gridDim.x * blockDim.y;
    const W *w = static_cast<const W *>(p.weight);
    const int c0 = threadIdx.x * VEC - shift_of<VEC, RAGGED>(first, p.dy_stride), across = blockDim.x * VEC;
    auto start = [&](unsigned r, const T *(&at)[3]) {
        at[0] = at_row(static_cast<const T *>(p.dy), r, p.dy_stride, c0);
        at[1] = at_row(static_cast<const T *>(p.h), r, p.h_stride, c0);
        at[2] = p.d_residual ? at_row(static_cast<const T *>(p.d_residual), r, p.d_residual_stride, c0) : nullptr;
    };
    Feed<T, VEC, NV, 3, RAGGED> feed;
    auto ask = [&](unsigned r) {
        const T *at[3];
        start(r, at);
        feed.ask(at, r < p.rows, c0, p.d, across);
    };
    if constexpr (FED) ask(first);
    Pack<W, VEC> wv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (c0 + i * across < p.d) wv[i] = load_weight<W, VEC, RAGGED>(w, c0 + i * across, p.d);
    int turn = 0;
    for (unsigned row = first; row < p.rows; row += step, turn ^= 1) {
        const float rstd = p.rstd[row];
        const T *at[3];
        if constexpr (FED) {
            feed.turn();
            ask(row + step);
            feed.wait();
        }
        if (RAGGED || !FED) start(row, at);
        Pack<T, VEC> own[3][FED ? 1 : NV] = {};     // without the feed a row stays in registers
        auto pack = [&](int k, int i) -> Pack<T, VEC> {
            if constexpr (!FED) return own[k][i];
            const int c = c0 + i * across;
            if constexpr (RAGGED) {
                if (!whole_pack<VEC, true>(c, p.d)) return load_part<T, VEC>(at[k] + i * across, c, p.d);
            }
            return feed.got(k, i);
        };
        if constexpr (!FED) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (c0 + i * across < p.d && at[k]) own[k][i] = load_some<T, VEC, RAGGED>(at[k] + i * across, c0 + i * across, p.d);
        }
        float2 dot = both(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (c0 + i * across >= p.d) continue;
            const Pack<T, VEC> dy = pack(0, i), h = pack(1, i);
            if constexpr (VEC == 1) {
                const float t = to_f32(dy.v[0]), n = to_f32(h.v[0]) * rstd;
                acc[i] = fmaf(t, n, acc[i]);
                dot.x = fmaf(t * to_f32(wv[i].v[0]), n, dot.x);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    const int k = i * VEC + j;
                    const float2 t = to_f32x2(&dy.v[j]), n = mul2(to_f32x2(&h.v[j]), both(rstd));
                    const float2 s = fma2(t, n, make_float2(acc[k], acc[k + 1]));
                    acc[k] = s.x, acc[k + 1] = s.y;
                    dot = fma2(mul2(t, to_f32x2(&wv[i].v[j])), n, dot);
                }
            }
        }
        // dx = rstd * (g - n * mean) = dy * (weight * rstd) - h * (rstd^2 * mean)
        const float mean = row_sum(dot.x + dot.y, buf[turn]) * p.per_d, back = -rstd * rstd * mean;
        T *dx = at_row(static_cast<T *>(p.dx), row, p.dx_stride, c0);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (c0 + i * across >= p.d) continue;
            const Pack<T, VEC> dy = pack(0, i), h = pack(1, i);
            Pack<T, VEC> add, o;
            if (p.d_residual) add = pack(2, i);
            if constexpr (VEC == 1) {
                float v = fmaf(to_f32(dy.v[0]), to_f32(wv[i].v[0]) * rstd, to_f32(h.v[0]) * back);
                if (p.d_residual) v += to_f32(add.v[0]);
                o.v[0] = from_f32<T>(v);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    float2 v = mul2(to_f32x2(&h.v[j]), both(back));
                    if (p.d_residual) v = add2(v, to_f32x2(&add.v[j]));
                    from_f32x2(&o.v[j], fma2(to_f32x2(&dy.v[j]), mul2(to_f32x2(&wv[i].v[j]), both(rstd)), v));
                }
            }
            store_some<T, VEC, RAGGED>(dx + i * across, o, c0 + i * across, p.d);
        }
    }
    if (!p.partial) return;
    float *out = p.partial + (long long)blockIdx.x * p.d;
    if (blockDim.y > 1) {
        // the sums of a block's rows first meet in shared memory, by columns and in the order of the warps: one partial row per block
        extern __shared__ __align__(16) uint8_t feed_memory[];
        float *sums = reinterpret_cast<float *>(feed_memory);
        asm volatile("cp.async.wait_all;" ::: "memory");        // nothing is on its way into that memory any more
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV * VEC; ++i) {
            const int c = c0 + i / VEC * across + i % VEC;
            if (c >= 0 && c < p.d) sums[threadIdx.y * p.d + c] = acc[i];
        }
        __syncthreads();
        for (int c = threadIdx.y * 32 + threadIdx.x; c < p.d; c += 32 * blockDim.y) {
            float t = 0.0f;
            for (int y = 0; y < blockDim.y; ++y) t += sums[y * p.d + c];
            out[c] = t;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = c0 + i * across;
        if constexpr (!RAGGED && VEC % 4 == 0) {
#pragma unroll
            for (int j = 0; j < VEC; j += 4)
                if (c < p.d) *reinterpret_cast<float4 *>(out + c + j) = make_float4(acc[i * VEC + j], acc[i * VEC + j + 1], acc[i * VEC + j + 2], acc[i * VEC + j + 3]);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (c + j >= 0 && c + j < p.d) out[c + j] = acc[i * VEC + j];
        }
    }
}

// In up to 64 registers (48, 40: 37, 46 us).
template <typename T, typename W, int VEC, int NV>
__global__ void __launch_bounds__(max_threads(VEC *NV)) add_norm_backward_kernel(const NormBackP p) { add_norm_backward_rows<T, W, VEC, NV, false>(p); }
// Ragged rows in 48, where 544 threads fit an SM twice (8000 x 4097: 93 us, in 64 142 us).
template <typename T, typename W, int VEC, int NV>
__global__ void __maxnreg__(VEC *NV <= 8 ? 48 : 128) add_norm_backward_ragged_kernel(const NormBackP p) { add_norm_backward_rows<T, W, VEC, NV, true>(p); }

// dweight[c] = sum of the partial rows: 32 columns per block, each by 32 threads with several loads in flight and then in one
// tree -- a fixed order.
__global__ void __launch_bounds__(1024) reduce_partials_kernel(const float *partial, int count, int d, float *dweight)
{
    __shared__ float buf[32][33];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < d) {
        int i = threadIdx.y;
        for (; i + 224 < count; i += 256) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = partial[(long long)(i + 32 * j) * d + c];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j & 3] += v[j];
        }
#pragma unroll 4
        for (; i < count; i += 32) s[0] += partial[(long long)i * d + c];
    }
    buf[threadIdx.y][threadIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    const float t = warp_sum(buf[threadIdx.x][threadIdx.y]);      // a warp per column
    const int out = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && out < d) dweight[out] = t;
}

struct SwigluP {
    unsigned rows;
    int f;
    const void *x;
    int8_t *q;
    float *scale;
    int x_stride, q_stride;
};

// g / (1 + exp(-g)) by the approximate power of two and reciprocal: relative error about 2^-22 + |g| 2^-24 before the rounding to
// 8 bits, 2^-17 at g = -80.  The full exponential and division take 20 instructions more per element, and the kernel would be bound by them,
// not by HBM.  From exp(-g) = 2^126 on (g < -87.3; infinite beyond -88.7) the reciprocal is 0, and so is the result, of less than 2^-119.
__device__ __forceinline__ float2 silu2(float2 g)
{
    const float2 p = mul2(g, both(-1.4426950408889634f));
    float2 e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(p.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(p.y));
    e = add2(e, both(1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
    return mul2(g, r);
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(swiglu_threads(VEC *NV)) swiglu_quant_kernel(const SwigluP p)
{
    __shared__ float buf[2][32];
    after_previous();
    may_follow();
    const unsigned step = gridDim.x * blockDim.y;
    unsigned row = blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.rows) return;
    const int c0 = threadIdx.x * VEC, across = blockDim.x * VEC;
    Pack<T, VEC> a[NV], b[NV];
    auto load = [&](unsigned r) {
        const T *g = at_row(static_cast<const T *>(p.x), r, p.x_stride, c0), *u = g + p.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (c0 + i * across < p.f) {
                a[i] = load_pack<T, VEC>(g + i * across);
                b[i] = load_pack<T, VEC>(u + i * across);
            }
    };
    load(row);
    for (int turn = 0; row < p.rows; row += step, turn ^= 1) {
        float v[NV * VEC], most = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (c0 + i * across >= p.f) continue;
            if constexpr (VEC == 1) {
                const float2 t = silu2(both(to_f32(a[i].v[0])));
                v[i] = t.x * to_f32(b[i].v[0]);
                most = max_abs(most, v[i]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    const float2 t = mul2(silu2(to_f32x2(&a[i].v[j])), to_f32x2(&b[i].v[j]));
                    v[i * VEC + j] = t.x, v[i * VEC + j + 1] = t.y;
                    most = max_abs(most, t);
                }
            }
        }
        if (row + step < p.rows) load(row + step);
        most = row_max(most, buf[turn]);
        const float factor = quant_factor(most);
        if (threadIdx.x == 0) p.scale[row] = quant_scale(most);
        const uint32_t keep = keep_mask(most);
        int8_t *q = at_row(p.q, row, p.q_stride, c0);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (c0 + i * across < p.f) store_quant<VEC, false>(q + i * across, v + i * VEC, factor, keep);
        }
    }
}

// Packs of VEC elements that a row can touch wherever it begins.
template <int VEC> int ragged_packs(int width) { return (width + 2 * (VEC - 1)) / VEC; }

// How a row of `width` elements is spread: threads per row, packs per thread, rows per block.
struct RowShape { int threads, packs, rows_per_block; };
int blocks_of(unsigned rows, const RowShape &s) { return (int)((rows - 1) / s.rows_per_block + 1); }

template <int VEC> RowShape row_shape(int rows, int width, int want_values, int (*most_threads)(int), bool ragged = false)
{
    const int packs = ragged ? ragged_packs<VEC>(width) : (width + VEC - 1) / VEC;
    // few rows leave SMs idle whatever the block is: the latency of one row counts, so a thread takes few values
    const int want = rows <= 296 ? 8 : want_values;
    auto threads = [&](int n) { return ((packs + n - 1) / n + 31) / 32 * 32; };
    auto next = [](int n) { return VEC >= 4 || n >= 32 ? 2 * n : 4 * n; };
    int nv = VEC >= 4 ? 1 : 2;
    while ((next(nv) * VEC <= want && packs > 32 * nv) || threads(nv) > most_threads(VEC * nv)) nv = next(nv);
    RowShape s = {threads(nv), nv, 1};
    if (s.threads == 32) s.rows_per_block = 8;
    return s;
}

int sm_count(int device)
{
    static std::atomic<int> known[64];
    std::atomic<int> &have = known[device & 63];
    int n = have.load(std::memory_order_relaxed);
    if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) == cudaSuccess && device < 64) have.store(n, std::memory_order_relaxed);
    return std::max(n, 1);
}

// As many blocks as the device holds at once, or as the rows need.  0: a CUDA call failed.
template <typename K> int resident(K kernel, int threads, int smem, int blocks, int device)
{
    if (blocks <= sm_count(device)) return blocks;
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess) return 0;
    return std::min(blocks, per_sm * sm_count(device));
}

// Ragged rows: a block's rows have to lie a multiple of VEC (8 at most) apart, unless each block has one row.
int whole_steps(int blocks, const RowShape &s, int rows, bool ragged) { return ragged && s.rows_per_block == 1 && blocks < rows && blocks > 8 ? blocks / 8 * 8 : blocks; }

template <typename K, typename P> int launch_rows(K kernel, const P &p, const RowShape &s, bool ragged, int device, cudaStream_t stream)
{
    const int blocks = whole_steps(resident(kernel, s.threads * s.rows_per_block, 0, blocks_of(p.rows, s), device), s, (int)p.rows, ragged);
    if (blocks < 1) return MOE_OVL_ERR_CUDA;
    return launch_behind(kernel, (unsigned)blocks, dim3(s.threads, s.rows_per_block), 0, 1, stream, p);
}

// `allowed`: whether this kernel has been allowed its shared memory on each device.
template <int VEC, int NV, typename T, typename K>
int launch_backward(K kernel, std::atomic<int> *allowed, const NormBackP &p, const RowShape &s, bool ragged, int device, cudaStream_t stream, int &blocks)
{
    const int threads = s.threads * s.rows_per_block;
    const int smem = std::max(BackFeed<T, VEC, NV>::ON ? 2 * BackFeed<T, VEC, NV>::THREAD_BYTES * threads : 0, s.rows_per_block > 1 ? s.rows_per_block * p.d * 4 : 0);
    if (smem > 46 * 1024 && (device > 63 || allowed[device].load(std::memory_order_relaxed) == 0)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024) != cudaSuccess) return MOE_OVL_ERR_CUDA;
        if (device <= 63) allowed[device].store(1, std::memory_order_relaxed);
    }
    blocks = resident(kernel, threads, smem, std::min(blocks_of(p.rows, s), NORM_PARTIALS), device);
    if (blocks < 1) return MOE_OVL_ERR_CUDA;
    blocks = whole_steps(blocks, s, (int)p.rows, ragged);
    return launch_behind(kernel, (unsigned)blocks, dim3(s.threads, s.rows_per_block), smem, 1, stream, p);
}

template <int N> struct Count { static constexpr int value = N; };
// Calls f with the number of packs as a constant: one of those that row_shape gives for some width, a kernel for each and no others.
template <typename F, int... N> int with_packs(int packs, std::integer_sequence<int, N...>, F f)
{
    int rc = MOE_OVL_ERR_UNSUPPORTED;
    ((packs == N ? (void)(rc = f(Count<N>())) : (void)0), ...);
    return rc;
}
template <int VEC> constexpr auto norm_packs()
{
    if constexpr (VEC == 8) return std::integer_sequence<int, 1, 4, 8>();
    else if constexpr (VEC == 4) return std::integer_sequence<int, 1, 2, 8, 16>();
    else return std::integer_sequence<int, 2, 8, 32, 64>();
}
template <int VEC> constexpr auto swiglu_packs()
{
    if constexpr (VEC == 8) return std::integer_sequence<int, 1, 2, 8>();
    else if constexpr (VEC == 4) return std::integer_sequence<int, 1, 2, 4, 16>();
    else if constexpr (VEC == 2) return std::integer_sequence<int, 2, 8, 32>();
    else return std::integer_sequence<int, 2, 8, 32, 64>();
}

// Calls f with the packs that the matrices allow, and whether rows are ragged in them: 16 bytes, or one element.  The widest rows fill a
// block's registers (512 threads of 64 elements) and leave no room for the one pack more that a ragged row can touch.
template <typename T, typename F> int with_ragged(bool wide, bool ragged, int width, F f)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    if (ragged_packs<VEC>(width) * VEC > MOE_OVL_MAX_ROW) ragged = false;
    if (wide) return f(Count<VEC>(), Count<0>());
    if (ragged) return f(Count<VEC>(), Count<1>());
    return f(Count<1>(), Count<0>());
}

// Calls f with the widest pack that the matrices allow: 16 bytes, a pair of 16-bit values, or one value.
template <typename T, typename F> int with_vec(bool wide, bool pairs, F f)
{
    if (wide) return f(Count<16 / (int)sizeof(T)>());
    if constexpr (sizeof(T) == 2) if (pairs) return f(Count<2>());
    return f(Count<1>());
}

bool rows_ok(const void *p, int64_t stride, int vec, int bytes) { return aligned(p, (size_t)vec * bytes) && stride % vec == 0; }

// Rows that do not overlap (or one row).
bool stride_ok(int64_t stride, int rows, int width) { return (rows <= 1 || stride >= width) && stride >= 0; }
// Kernels take strides of 31 bits (offsets are 64 bits wide).
bool fits_int(int64_t a, int64_t b = 0, int64_t c = 0, int64_t d = 0, int64_t e = 0) { return std::max({a, b, c, d, e}) <= 0x7fffffff; }

}  // namespace

extern "C" int moe_ovl_add_norm(const moe_ovl_norm_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->d < 1 || a->flags != 0) return MOE_OVL_ERR_INVALID_ARG;
    if (!known_dtype(a->dtype) || (a->weight_dtype != a->dtype && a->weight_dtype != MOE_OVL_F32) || !(a->eps >= 0.0f))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->d > MOE_OVL_MAX_ROW) return MOE_OVL_ERR_UNSUPPORTED;
    if ((a->q == nullptr) != (a->scale == nullptr) || !stride_ok(a->x_stride, a->rows, a->d) ||
        (a->residual && !stride_ok(a->residual_stride, a->rows, a->d)) ||
        (a->residual_out && !stride_ok(a->residual_out_stride, a->rows, a->d)) ||
        (a->y && !stride_ok(a->y_stride, a->rows, a->d)) || (a->q && !stride_ok(a->q_stride, a->rows, a->d)))
        return MOE_OVL_ERR_INVALID_ARG;
    if (!fits_int(a->x_stride, a->residual_stride, a->residual_out_stride, a->y_stride, a->q_stride)) return MOE_OVL_ERR_UNSUPPORTED;
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->dtype), ws = dtype_bytes(a->weight_dtype);
    if (!a->x || !a->weight || !aligned(a->x, es) || !aligned(a->residual, es) || !aligned(a->residual_out, es) || !aligned(a->y, es) ||
        !aligned(a->weight, ws) || !aligned(a->scale, 4) || !aligned(a->rstd, 4))
        return MOE_OVL_ERR_INVALID_ARG;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const NormP p = {(unsigned)a->rows, a->d, 1.0f / (float)a->d, a->eps, a->x, a->residual, a->weight, a->residual_out, a->y, a->q, a->scale, a->rstd,
                     (int)a->x_stride, (int)a->residual_stride, (int)a->residual_out_stride, (int)a->y_stride, (int)a->q_stride};
    auto fits = [&](int vec) {
        return a->d % vec == 0 && rows_ok(a->x, a->x_stride, vec, es) && aligned(a->weight, (size_t)vec * ws) &&
               (!a->residual || rows_ok(a->residual, a->residual_stride, vec, es)) &&
               (!a->residual_out || rows_ok(a->residual_out, a->residual_out_stride, vec, es)) &&
               (!a->y || rows_ok(a->y, a->y_stride, vec, es)) && (!a->q || rows_ok(a->q, a->q_stride, vec, 1));
    };
    auto agree = [&](int vec) {
        auto like_x = [&](const void *m, int64_t stride, int bytes) { return !m || (aligned(m, (size_t)vec * bytes) && (stride - a->x_stride) % vec == 0); };
        return like_x(a->x, a->x_stride, es) && like_x(a->residual, a->residual_stride, es) && like_x(a->residual_out, a->residual_out_stride, es) &&
               like_x(a->y, a->y_stride, es) && like_x(a->q, a->q_stride, 1);
    };
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto w, auto v, auto r) {
            using W = decltype(w);
            constexpr int VEC = decltype(v)::value;
            constexpr bool RAGGED = decltype(r)::value != 0;
            const RowShape s = row_shape<VEC>(a->rows, p.d, VEC >= 4 ? VEC : 8, max_threads, RAGGED);
            return with_packs(s.packs, norm_packs<VEC>(), [&](auto n) {
                constexpr int NV = decltype(n)::value;
                // An 8-bit output alone: blocks per SM count (16384 x 4096, bf16: 71 us in 40 registers, 80 us in 64).  With an output in the type of x the
                // writes are what bounds it, and fewer blocks write better (85 us in 64, 92 us in 40).  f32 rows of 4097 to 8192 columns spill in 40.
                const auto kernel = p.q && !p.y ? add_norm_lean_kernel<T, W, VEC, NV, RAGGED> : add_norm_kernel<T, W, VEC, NV, RAGGED>;
                return launch_rows(kernel, p, s, RAGGED, a->device, static_cast<cudaStream_t>(a->stream));
            });
        };
        return with_ragged<T>(fits(16 / es), agree(16 / es), a->d, [&](auto v, auto r) {
            return a->weight_dtype == a->dtype ? launch(T(), v, r) : launch(0.0f, v, r);
        });
    });
}

extern "C" int moe_ovl_add_norm_workspace_bytes(int32_t rows, int32_t d, size_t *bytes)
{
    if (!bytes || rows < 0 || d < 1) return MOE_OVL_ERR_INVALID_ARG;
    if (d > MOE_OVL_MAX_ROW) return MOE_OVL_ERR_UNSUPPORTED;
    *bytes = (size_t)(rows < NORM_PARTIALS ? rows : NORM_PARTIALS) * d * 4;
    return MOE_OVL_OK;
}

extern "C" int moe_ovl_add_norm_backward(const moe_ovl_norm_backward_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->d < 1) return MOE_OVL_ERR_INVALID_ARG;
    if (!known_dtype(a->dtype) || (a->weight_dtype != a->dtype && a->weight_dtype != MOE_OVL_F32)) return MOE_OVL_ERR_INVALID_ARG;
    if (a->d > MOE_OVL_MAX_ROW) return MOE_OVL_ERR_UNSUPPORTED;
    if (!stride_ok(a->dy_stride, a->rows, a->d) || !stride_ok(a->h_stride, a->rows, a->d) || !stride_ok(a->dx_stride, a->rows, a->d) ||
        (a->d_residual && !stride_ok(a->d_residual_stride, a->rows, a->d)))
        return MOE_OVL_ERR_INVALID_ARG;
    if (!fits_int(a->dy_stride, a->h_stride, a->d_residual_stride, a->dx_stride)) return MOE_OVL_ERR_UNSUPPORTED;
    const int es = dtype_bytes(a->dtype), ws = dtype_bytes(a->weight_dtype);
    if (a->rows > 0 && (!a->dy || !a->h || !a->weight || !a->rstd || !a->dx || !aligned(a->dy, es) || !aligned(a->h, es) ||
                        !aligned(a->d_residual, es) || !aligned(a->dx, es) || !aligned(a->weight, ws) || !aligned(a->rstd, 4)))
        return MOE_OVL_ERR_INVALID_ARG;
    if (!aligned(a->dweight, 4)) return MOE_OVL_ERR_INVALID_ARG;
    size_t need = 0;
    moe_ovl_add_norm_workspace_bytes(a->rows, a->d, &need);
    if (a->dweight && need > 0 && (!a->workspace || !aligned(a->workspace, 16) || a->workspace_bytes < need)) return MOE_OVL_ERR_WORKSPACE;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    if (a->rows == 0) {
        if (!a->dweight) return MOE_OVL_OK;
        return cudaMemsetAsync(a->dweight, 0, (size_t)a->d * 4, stream) == cudaSuccess ? MOE_OVL_OK : MOE_OVL_ERR_CUDA;
    }
    const NormBackP p = {(unsigned)a->rows, a->d, 1.0f / (float)a->d, a->dy, a->h, a->weight, a->d_residual, a->rstd, a->dx,
                   a->dweight ? static_cast<float *>(a->workspace) : nullptr, (int)a->dy_stride, (int)a->h_stride,
                   (int)a->d_residual_stride, (int)a->dx_stride};
    auto fits = [&](int vec) {
        return a->d % vec == 0 && rows_ok(a->dy, a->dy_stride, vec, es) && rows_ok(a->h, a->h_stride, vec, es) &&
               rows_ok(a->dx, a->dx_stride, vec, es) && aligned(a->weight, (size_t)vec * ws) &&
               (!a->d_residual || rows_ok(a->d_residual, a->d_residual_stride, vec, es));
    };
    auto agree = [&](int vec) {
        auto like_dy = [&](const void *m, int64_t stride) { return !m || (aligned(m, (size_t)vec * es) && (stride - a->dy_stride) % vec == 0); };
        return like_dy(a->dy, a->dy_stride) && like_dy(a->h, a->h_stride) && like_dy(a->d_residual, a->d_residual_stride) && like_dy(a->dx, a->dx_stride);
    };
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto w, auto v, auto r) {
            using W = decltype(w);
            constexpr int VEC = decltype(v)::value;
            constexpr bool RAGGED = decltype(r)::value != 0;
            const RowShape s = row_shape<VEC>(a->rows, p.d, 8, max_threads, RAGGED);
            return with_packs(s.packs, norm_packs<VEC>(), [&](auto n) {
                constexpr int NV = decltype(n)::value;
                int blocks = 0;
                static std::atomic<int> allowed[64];
                void (*kernel)(NormBackP);
                if constexpr (RAGGED) kernel = add_norm_backward_ragged_kernel<T, W, VEC, NV>;
                else kernel = add_norm_backward_kernel<T, W, VEC, NV>;
                const int rc = launch_backward<VEC, NV, T>(kernel, allowed, p, s, RAGGED, a->device, stream, blocks);
                if (rc != MOE_OVL_OK || !p.partial) return rc;
                reduce_partials_kernel<<<(p.d + 31) / 32, dim3(32, 32), 0, stream>>>(p.partial, blocks, p.d, a->dweight);
                return launched();
            });
        };
        return with_ragged<T>(fits(16 / es), agree(16 / es), a->d, [&](auto v, auto r) {
            return a->weight_dtype == a->dtype ? launch(T(), v, r) : launch(0.0f, v, r);
        });
    });
}

extern "C" int moe_ovl_swiglu_quant(const moe_ovl_swiglu_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->f < 1 || a->flags != 0) return MOE_OVL_ERR_INVALID_ARG;
    if (!known_dtype(a->dtype)) return MOE_OVL_ERR_INVALID_ARG;
    if (a->f > MOE_OVL_MAX_ROW) return MOE_OVL_ERR_UNSUPPORTED;
    if (!stride_ok(a->gate_up_stride, a->rows, 2 * a->f) || !stride_ok(a->q_stride, a->rows, a->f)) return MOE_OVL_ERR_INVALID_ARG;
    if (!fits_int(a->gate_up_stride, a->q_stride)) return MOE_OVL_ERR_UNSUPPORTED;
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->dtype);
    if (!a->gate_up || !a->q || !a->scale || !aligned(a->gate_up, es) || !aligned(a->scale, 4)) return MOE_OVL_ERR_INVALID_ARG;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const SwigluP p = {(unsigned)a->rows, a->f, a->gate_up, a->q, a->scale, (int)a->gate_up_stride, (int)a->q_stride};
    auto fits = [&](int vec) { return a->f % vec == 0 && rows_ok(a->gate_up, a->gate_up_stride, vec, es) && rows_ok(a->q, a->q_stride, vec, 1); };
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto v) {
            constexpr int VEC = decltype(v)::value;
            const RowShape s = row_shape<VEC>(a->rows, p.f, 16, swiglu_threads);
            return with_packs(s.packs, swiglu_packs<VEC>(), [&](auto n) {
                constexpr int NV = decltype(n)::value;
                return launch_rows(swiglu_quant_kernel<T, VEC, NV>, p, s, false, a->device, static_cast<cudaStream_t>(a->stream));
            });
        };
        return with_vec<T>(fits(16 / es), fits(2), launch);
    });
}
