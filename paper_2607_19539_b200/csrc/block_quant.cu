// Values in 8-bit floats (e4m3) with a scale for each block of 128, or for each 128 x 128 (moe_ovl_block_quant in include/moe_ovl.h):
//   scale = max|v| / 448,  q = v / scale = v * 448 / max|v|, to the nearest, ties to even.
//
// 16-bit values lie half-way between two of e4m3's steps often (max|v| = 1.75 puts one in sixteen there), so the quotient is rounded as
// division rounds it: a product with a rounded 448 / max|v| would send ties either way.  The division is one by Newton's step on the remainder (P. Markstein, Computation
// of elementary functions on the IBM RISC System/6000 processor, 1990): with r the reciprocal of d, q0 = n r and q = q0 + r (n - d q0), the
// remainder formed exactly by a fused operation.  n and d are scaled by a power of two, d into [2, 4), so that nothing overflows.
#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "opcommon.cuh"

using namespace moe_ovl;

namespace {

constexpr int BQ_BLOCK = 128;
constexpr float BQ_LARGEST = 448.0f;
constexpr float BQ_TINY = 7.8886090522101181e-31f;      // 2^-100: below it a block is zeros

// What a block's values are divided by.
struct Divisor {
    float2 factor, minus_d, inverse;         // 448 * 2^s; -max * 2^s; 1 / (max * 2^s)
    float scale;
    bool none;                               // all zeros, or not a number: q is 0
};
__device__ __forceinline__ Divisor divisor_of(float most)
{
    Divisor d;
    d.none = !(most >= BQ_TINY && most <= 3.402823466e38f);
    const bool low = most < BQ_TINY;
    if (d.none) most = 1.0f;
    // by the same step: the reciprocal of 448 is a constant
    const float s0 = most * (1.0f / BQ_LARGEST), scale = fmaf(fmaf(-s0, BQ_LARGEST, most), 1.0f / BQ_LARGEST, s0);
    d.scale = low ? 0.0f : d.none ? __int_as_float(0x7fffffff) : scale;
    // 2^(1 - exponent of most): the exponent field is 27 .. 254, so that of the power 228 .. 1
    const float power = __uint_as_float((255u - (__float_as_uint(most) >> 23)) << 23);
    const float whole = most * power;
    d.factor = both(BQ_LARGEST * power);
    d.minus_d = both(-whole);
    float inverse;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(whole));
    inverse = fmaf(inverse, fmaf(-whole, inverse, 1.0f), inverse);
    d.inverse = both(inverse);
    return d;
}
template <typename T> __device__ __forceinline__ float2 divided(float2 v, const Divisor &d)
{
    const float2 n = mul2(v, d.factor);                  // exact for 16-bit values: 11 + 3 bits
    const float2 q = mul2(n, d.inverse);
    float2 rest = fma2(q, d.minus_d, n);
    if (sizeof(T) == 4) rest = add2(rest, fma2(v, d.factor, make_float2(-n.x, -n.y)));       // what rounding took off n
    return fma2(rest, d.inverse, q);
}
__device__ __forceinline__ uint16_t rounded(float2 v) { return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3); }

// g / (1 + exp(-g)) * u; exp(-g) = 2^(-g / ln 2).
__device__ __forceinline__ float2 gate(float2 g, float2 u)
{
    const float2 power = mul2(g, both(-1.4426950408889634f));
    float2 e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(power.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(power.y));
    e = add2(e, both(1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.y) : "f"(e.y));
    return mul2(mul2(g, s), u);
}

struct BqP {
    const void *x;
    uint8_t *q;
    float *scale;
    long long x_stride, q_stride, x_far, q_far;
    int rows, k, blocks;
    unsigned units;                          // rows * blocks of this launch
    unsigned long long magic;                // floor(2^64 / blocks) + 1: 32-bit quotients by blocks
};

// A pack of VEC values of which `left` exist.  EVEN: all of them or none, which takes no branch.
template <typename T, int VEC, bool EVEN> __device__ __forceinline__ Pack<T, VEC> load_some(const T *p, int left)
{
    Pack<T, VEC> r = {};
    if (EVEN) {
        if (left > 0) r = load_pack<T, VEC>(p);
    } else if (left >= VEC) {
        r = load_pack<T, VEC>(p);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) r.v[i] = p[i];
    }
    return r;
}
// A pack's values in 8 bits, of which `left` exist.
template <typename T, int VEC, bool EVEN> __device__ __forceinline__ void store_rounded(uint8_t *q, const float2 (&v)[(VEC + 1) / 2], const Divisor &d, int left)
{
    uint32_t w[(VEC + 3) / 4] = {};
    if (!d.none) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
            w[i / 4] = rounded(divided<T>(v[i / 2], d));
            if (VEC > 2) w[i / 4] |= (uint32_t)rounded(divided<T>(v[(i / 2 + 1) % ((VEC + 1) / 2)], d)) << 16;
        }
    }
    if (VEC > 1 && (EVEN || left >= VEC)) {
        if (left > 0) {
            if (VEC == 8) *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[VEC / 8]);
            else *reinterpret_cast<uint32_t *>(q) = w[0];
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) q[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}
// A pack as floats (an odd one out has a 0 beside it).
template <typename T, int VEC> __device__ __forceinline__ void floats(const Pack<T, VEC> &a, float2 (&v)[(VEC + 1) / 2])
{
#pragma unroll
    for (int e = 0; e < VEC; e += 2) v[e / 2] = VEC == 1 ? make_float2(to_f32(a.v[0]), 0.0f) : to_f32x2(&a.v[e]);
}

// Below this gate() loses what a large value leaves of itself: 1 / (1 + exp(-g)) ends as a normal number at -87.3.  Of f16 no value is large enough to matter.
constexpr float BQ_FAR = -86.0f;
// The smallest of a pack's gates and `low`.
template <typename T, int VEC> __device__ __forceinline__ T lowest(T low, const Pack<T, VEC> &g)
{
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        if constexpr (std::is_same<T, float>::value) low = fminf(low, g.v[e]);
        else low = __hmin(low, g.v[e]);
    }
    return low;
}
template <int VEC> __device__ __forceinline__ __nv_bfloat162 lowest(__nv_bfloat162 low, const Pack<__nv_bfloat16, VEC> &g)
{
#pragma unroll
    for (int e = 0; e < VEC; e += 2) low = __hmin2(low, *reinterpret_cast<const __nv_bfloat162 *>(&g.v[e]));
    return low;
}

constexpr int BQ_THREADS = 256, BQ_RESIDENT = 8;     // blocks per SM

// Blocks of 1 x 128.  LANES lanes work on a block, PER packs of VEC values each; a group of lanes has the loads of AHEAD neighbouring blocks under way.
template <typename T, int VEC, bool GATED> struct BqShape {
    static constexpr int LANES = VEC == 1 ? 32 : BQ_BLOCK / VEC / 2, PER = BQ_BLOCK / VEC / LANES, AHEAD = VEC == 1 ? 1 : 2;
};
// What a gate leaves of a value, from far below zero too: there 1 + exp(-g) is exp(-g), and g * 2^(126 + g / ln 2) * u * 2^-126 is taken in an order in which nothing overflows and nothing that a block keeps
// falls below the normal numbers.
__device__ __forceinline__ float any_gate(float g, float u)
{
    if (!(g < BQ_FAR)) return gate(make_float2(g, g), make_float2(u, u)).x;
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(g, 1.4426950408889634f, 126.0f)));
    return g * e * (u * 5.4210108624275222e-20f) * 2.1684043449710089e-19f;      // 2^-64, 2^-62
}
// Gated blocks that have such gates, once more and value by value: `count` of them from `u` on, by LANES lanes.  Out of the way of the others, which would pay for it with registers (8192 x 14336, bf16: 130 us
// with the choice inside their loop, 98 with a vote at its end and 98 without any).
template <typename T, int LANES> __device__ __noinline__ void far_blocks(BqP p, unsigned u, int count, int lane)
{
    __syncwarp();                            // behind what the lanes have stored
    for (; count > 0; --count, ++u) {
        const unsigned row = p.blocks == 1 ? u : (unsigned)__umul64hi(p.magic, u);
        const int col = (int)(u - row * (unsigned)p.blocks) * BQ_BLOCK, end = u < p.units ? min(col + BQ_BLOCK, p.k) : 0;
        const T *x = static_cast<const T *>(p.x) + (long long)row * p.x_stride;
        float most = 0.0f;
        for (int c = col + lane; c < end; c += LANES) most = max_abs(most, any_gate(to_f32(x[c]), to_f32(x[c + p.k])));
        for (int o = LANES / 2; o > 0; o >>= 1) most = max_abs(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (end == 0) continue;
        const Divisor d = divisor_of(most);
        if (lane == 0) p.scale[u] = d.scale;
        uint8_t *q = p.q + (long long)row * p.q_stride;
        for (int c = col + lane; c < end; c += LANES) {
            const float v = any_gate(to_f32(x[c]), to_f32(x[c + p.k]));
            q[c] = d.none ? 0 : (uint8_t)rounded(divided<T>(make_float2(v, 0.0f), d));
        }
    }
}
// Bound by HBM (8192 x 14336, bf16: 58 us, 6.1 TB/s; with the gate, whose instructions come next, 98-101 us, 5.9 TB/s; f32 159).  Eight lanes for a block of 128 values, not sixteen with a pack each: the maximum's shuffles and what a block
// costs besides its values weigh half as much (96 -> 58 us).  Rows that begin anywhere go element by element (8192 x 14335: 153 us, gated 219-230).
template <typename T, int VEC, bool GATED, bool EVEN>
__global__ void __launch_bounds__(BQ_THREADS)
block_quant_kernel(const BqP p)
{
    using Shape = BqShape<T, VEC, GATED>;
    constexpr int LANES = Shape::LANES, PER = Shape::PER, AHEAD = Shape::AHEAD, HALF = (VEC + 1) / 2;
    const int lane = threadIdx.x % LANES;
    const unsigned group = blockIdx.x * (BQ_THREADS / LANES) + threadIdx.x / LANES, step = gridDim.x * (BQ_THREADS / LANES) * AHEAD;
    after_previous();
    may_follow();
    // whole warps stay: the shuffles need all of their lanes
    const unsigned own = group * AHEAD, first = own - threadIdx.x % 32 / LANES * AHEAD;
    for (unsigned done = 0; first + done < p.units; done += step) {
        const unsigned u = own + done, row0 = p.blocks == 1 ? u : (unsigned)__umul64hi(p.magic, u), block0 = u - row0 * (unsigned)p.blocks;
        Pack<T, VEC> a[AHEAD][PER], b[GATED ? AHEAD : 1][PER];
        constexpr bool FAR = GATED && !std::is_same<T, __half>::value;
        using Low = std::conditional_t<std::is_same<T, __nv_bfloat16>::value && VEC % 2 == 0, __nv_bfloat162, T>;
        Low low = {};
        unsigned row = row0, block = block0;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int col = (int)block * BQ_BLOCK + lane * VEC, left = u + i < p.units ? p.k - col : 0;
            const T *at = static_cast<const T *>(p.x) + (long long)row * p.x_stride + col;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                a[i][j] = load_some<T, VEC, EVEN>(at + j * LANES * VEC, left - j * LANES * VEC);
                if (GATED) b[i][j] = load_some<T, VEC, EVEN>(at + j * LANES * VEC + p.k, left - j * LANES * VEC);
            }
            if (++block == (unsigned)p.blocks) block = 0, ++row;
        }
        row = row0, block = block0;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float2 v[PER][HALF];
            float most = 0.0f;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                floats(a[i][j], v[j]);
                if (GATED) {
                    if constexpr (FAR) low = lowest(low, a[i][j]);
                    float2 up[HALF];
                    floats(b[i][j], up);
#pragma unroll
                    for (int e = 0; e < HALF; ++e) v[j][e] = gate(v[j][e], up[e]);
                }
#pragma unroll
                for (int e = 0; e < HALF; ++e) most = max_abs(most, v[j][e]);
            }
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) most = max_abs(most, __shfl_xor_sync(0xffffffffu, most, o));
            if (u + i < p.units) {
                const Divisor d = divisor_of(most);
                if (lane == 0) p.scale[u + i] = d.scale;
                const int col = (int)block * BQ_BLOCK + lane * VEC;
                uint8_t *q = p.q + (long long)row * p.q_stride + col;
#pragma unroll
                for (int j = 0; j < PER; ++j) store_rounded<T, VEC, EVEN>(q + j * LANES * VEC, v[j], d, p.k - col - j * LANES * VEC);
            }
            if (++block == (unsigned)p.blocks) block = 0, ++row;
        }
        if constexpr (FAR) {
            float least;
            if constexpr (std::is_same<Low, __nv_bfloat162>::value) least = fminf(__low2float(low), __high2float(low));
            else least = to_f32(low);
            if (__any_sync(0xffffffffu, least < BQ_FAR)) far_blocks<T, LANES>(p, u, AHEAD, lane);
        }
    }
}

// Blocks of 128 x 128, one thread block each: the values stay in registers between the maximum and the division.  Bound by HBM (8 x 2816 x 2048, f32: 38 us, 6.1 TB/s).
template <typename T, int VEC, bool EVEN>
__global__ void __launch_bounds__(BQ_THREADS)
block_quant_tiles_kernel(const BqP p)
{
    constexpr int LANES = BQ_BLOCK / VEC, ROWS = BQ_THREADS / LANES, PACKS = BQ_BLOCK / ROWS;
    __shared__ float s_most[BQ_THREADS / 32];
    after_previous();
    may_follow();
    const int col = (int)blockIdx.x * BQ_BLOCK + (int)(threadIdx.x % LANES) * VEC, row0 = (int)blockIdx.y * BQ_BLOCK + (int)(threadIdx.x / LANES);
    const T *x = static_cast<const T *>(p.x) + blockIdx.z * p.x_far + col;
    uint8_t *q = p.q + blockIdx.z * p.q_far + col;
    Pack<T, VEC> a[PACKS];
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
        const long long row = row0 + i * ROWS;
        a[i] = load_some<T, VEC, EVEN>(x + row * p.x_stride, row < p.rows ? p.k - col : 0);
    }
#pragma unroll
    for (int i = 0; i < PACKS; ++i)
#pragma unroll
        for (int e = 0; e < (VEC + 1) / 2; ++e) {
            float2 v[(VEC + 1) / 2];
            floats(a[i], v);
            most = max_abs(most, v[e]);
        }
    most = warp_max(most);
    if (threadIdx.x % 32 == 0) s_most[threadIdx.x / 32] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < BQ_THREADS / 32; ++i) most = max_abs(most, s_most[i]);
    const Divisor d = divisor_of(most);
    if (threadIdx.x == 0) p.scale[((long long)blockIdx.z * gridDim.y + blockIdx.y) * p.blocks + blockIdx.x] = d.scale;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
        const long long row = row0 + i * ROWS;
        float2 v[(VEC + 1) / 2];
        floats(a[i], v);
        if (row < p.rows) store_rounded<T, VEC, EVEN>(q + row * p.q_stride, v, d, p.k - col);
    }
}

template <typename T, int VEC, bool GATED, bool EVEN> int launch_rows(BqP p, cudaStream_t stream)
{
    constexpr int PER_BLOCK = BQ_THREADS / BqShape<T, VEC, GATED>::LANES * BqShape<T, VEC, GATED>::AHEAD;
    // units are counted in 32 bits: very many rows go in several launches
    const int at_once = (int)std::min<long long>(p.rows, (1ll << 30) / p.blocks);
    const int rows = p.rows;
    p.magic = ~0ull / (unsigned)p.blocks + 1;
    for (long long done = 0; done < rows; done += at_once) {
        BqP part = p;
        part.rows = (int)std::min<long long>(at_once, rows - done);
        part.units = (unsigned)part.rows * (unsigned)p.blocks;
        part.x = static_cast<const T *>(p.x) + done * p.x_stride;
        part.q = p.q + done * p.q_stride;
        part.scale = p.scale + done * p.blocks;
        const unsigned blocks = std::min<unsigned>((part.units + PER_BLOCK - 1) / PER_BLOCK, 148 * BQ_RESIDENT);
        const int rc = launch_behind(block_quant_kernel<T, VEC, GATED, EVEN>, blocks, dim3(BQ_THREADS), 0, 1, stream, part);
        if (rc != MOE_OVL_OK) return rc;
    }
    return MOE_OVL_OK;
}

template <typename T, int VEC, bool EVEN> int launch_tiles(const BqP &p, int depth, cudaStream_t stream)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.blocks, (unsigned)((p.rows - 1) / BQ_BLOCK + 1), (unsigned)depth);
    cfg.blockDim = dim3(BQ_THREADS);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, block_quant_tiles_kernel<T, VEC, EVEN>, p) == cudaSuccess ? MOE_OVL_OK : MOE_OVL_ERR_CUDA;
}

}  // namespace

extern "C" int moe_ovl_block_quant(const moe_ovl_block_quant_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->depth < 1 || a->rows < 0 || a->k < 1 || !known_dtype(a->dtype) || (a->gated & ~1) != 0 ||
        (a->tiles & ~1) != 0 || (a->tiles && a->gated) || (!a->tiles && a->depth != 1) || a->flags != 0)
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->k > MOE_OVL_MAX_MATMUL || (a->tiles && (a->rows > 65535 * BQ_BLOCK || a->depth > 65535))) return MOE_OVL_ERR_UNSUPPORTED;
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->dtype);
    const long long width = a->gated ? 2ll * a->k : a->k;
    if (!a->x || !a->q || !a->scale || !aligned(a->x, es) || !aligned(a->scale, 4) || (a->rows > 1 && (a->x_stride < width || a->q_stride < a->k)) ||
        (a->depth > 1 && (a->x_far < 1 || a->q_far < 1)))
        return MOE_OVL_ERR_INVALID_ARG;
    if (std::max(a->x_stride, a->q_stride) > 0x7fffffff) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    BqP p = {};
    p.x = a->x, p.q = static_cast<uint8_t *>(a->q), p.scale = a->scale, p.x_stride = a->x_stride, p.q_stride = a->q_stride;
    p.x_far = a->depth > 1 ? a->x_far : 0, p.q_far = a->depth > 1 ? a->q_far : 0;
    p.rows = a->rows, p.k = a->k, p.blocks = (a->k - 1) / BQ_BLOCK + 1;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / sizeof(T);
        // packs of 16 bytes in, VEC bytes out, wherever a row, a matrix or the gate's other half begins
        const bool rows_fit = a->rows == 1 || (a->x_stride % VEC == 0 && a->q_stride % VEC == 0);
        const bool packs = aligned(a->x, 16) && aligned(a->q, VEC) && rows_fit && p.x_far % VEC == 0 && p.q_far % VEC == 0 && (!a->gated || a->k % VEC == 0);
        const bool even = a->k % VEC == 0;
        if (a->tiles) return !packs ? launch_tiles<T, 1, true>(p, a->depth, stream) : even ? launch_tiles<T, VEC, true>(p, a->depth, stream) : launch_tiles<T, VEC, false>(p, a->depth, stream);
        if (a->gated) return packs ? launch_rows<T, VEC, true, true>(p, stream) : launch_rows<T, 1, true, true>(p, stream);
        return !packs ? launch_rows<T, 1, false, true>(p, stream) : even ? launch_rows<T, VEC, false, true>(p, stream) : launch_rows<T, VEC, false, false>(p, stream);
    });
}
