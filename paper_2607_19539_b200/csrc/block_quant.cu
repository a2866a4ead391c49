// Values in 8-bit floats (e4m3) with a scale for each block of 128, or for each 128 x 128 (moe_ovl_block_quant in include/moe_ovl.h):
//   scale = max|v| / 448,  q = v / scale = v * 448 / max|v|, to the nearest, ties to even.
//
// 16-bit values lie half-way between two of e4m3's steps often (max|v| = 1.75 puts one in sixteen there), so the quotient is rounded as
// division rounds it: a product with a rounded 448 / max|v| would send ties either way.  The division is one by Newton's step on the remainder (P. Markstein, Computation
// of elementary functions on the IBM RISC System/6000 processor, 1990): with r the rounded reciprocal of d, q0 = n r and q = q0 + r (n - d q0), the
// remainder formed exactly by a fused operation.  n and d are scaled by a power of two, d into [2, 4), so that nothing overflows.
#include <cuda_fp8.h>

#include <algorithm>

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
    d.scale = most < BQ_TINY ? 0.0f : most > 3.402823466e38f ? __int_as_float(0x7fffffff) : __fdiv_rn(most, BQ_LARGEST);
    if (d.none) most = 1.0f;
    // 2^(1 - exponent of most): the exponent field is 27 .. 254, so that of the power 228 .. 1
    const float power = __uint_as_float((255u - (__float_as_uint(most) >> 23)) << 23);
    const float whole = most * power;
    d.factor = both(BQ_LARGEST * power);
    d.minus_d = both(-whole);
    d.inverse = both(__frcp_rn(whole));
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

__device__ __forceinline__ float2 gate(float2 g, float2 u)
{
    return make_float2(g.x / (1.0f + __expf(-g.x)) * u.x, g.y / (1.0f + __expf(-g.y)) * u.y);
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

// A pack of VEC values of which `left` exist.
template <typename T, int VEC> __device__ __forceinline__ Pack<T, VEC> load_some(const T *p, int left)
{
    if (left >= VEC) return load_pack<T, VEC>(p);
    Pack<T, VEC> r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = i < left ? p[i] : from_f32<T>(0.0f);
    return r;
}
template <int VEC> __device__ __forceinline__ void store_some(uint8_t *q, const uint8_t (&v)[VEC], int left)
{
    if (left >= VEC && VEC > 1) {
        Pack<uint8_t, VEC> p;
#pragma unroll
        for (int i = 0; i < VEC; ++i) p.v[i] = v[i];
        store_pack(q, p);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) q[i] = v[i];
    }
}
// A pack's values in 8 bits.
template <typename T, int VEC> __device__ __forceinline__ void quantise(const float (&v)[VEC], const Divisor &d, uint8_t (&q)[VEC])
{
    if constexpr (VEC == 1) {
        q[0] = (uint8_t)(d.none ? 0 : rounded(divided<T>(make_float2(v[0], 0.0f), d)));
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
            const uint16_t two = d.none ? (uint16_t)0 : rounded(divided<T>(make_float2(v[i], v[i + 1]), d));
            q[i] = (uint8_t)two, q[i + 1] = (uint8_t)(two >> 8);
        }
    }
}

constexpr int BQ_THREADS = 256;

// Blocks of 1 x 128.  LANES lanes work on a block, PER packs of VEC values each; a thread has AHEAD blocks' loads under way.
template <typename T, int VEC, bool GATED>
__global__ void __launch_bounds__(BQ_THREADS)
block_quant_kernel(const BqP p)
{
    constexpr int LANES = BQ_BLOCK / VEC < 32 ? BQ_BLOCK / VEC : 32, PER = BQ_BLOCK / VEC / LANES, AHEAD = VEC > 1 ? (GATED ? 2 : 4) : 1;
    const int lane = threadIdx.x % LANES;
    const unsigned group = blockIdx.x * (BQ_THREADS / LANES) + threadIdx.x / LANES, groups = gridDim.x * (BQ_THREADS / LANES);
    after_previous();
    may_follow();
    const T *x = static_cast<const T *>(p.x);
    // whole warps stay: the shuffles below need all of their lanes
    for (unsigned long long u0 = group; u0 - threadIdx.x % 32 / LANES < p.units; u0 += (unsigned long long)groups * AHEAD) {
        Pack<T, VEC> a[AHEAD][PER], b[AHEAD][PER];
        unsigned row[AHEAD], block[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const unsigned long long u = u0 + (unsigned long long)groups * i;
            row[i] = (unsigned)__umul64hi(p.magic, u), block[i] = (unsigned)u - row[i] * (unsigned)p.blocks;
            if (p.blocks == 1) row[i] = (unsigned)u, block[i] = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int col = (int)block[i] * BQ_BLOCK + (j * LANES + lane) * VEC, left = u < p.units ? p.k - col : 0;
                const T *at = x + (long long)row[i] * p.x_stride + col;
                a[i][j] = load_some<T, VEC>(at, left);
                if (GATED) b[i][j] = load_some<T, VEC>(at + p.k, left);
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float v[PER][VEC], most = 0.0f;
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[j][e] = to_f32(a[i][j].v[e]);
                    if (GATED) v[j][e] = gate(make_float2(v[j][e], 0.0f), make_float2(to_f32(b[i][j].v[e]), 0.0f)).x;
                    most = max_abs(most, v[j][e]);
                }
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) most = max_abs(most, __shfl_xor_sync(0xffffffffu, most, o));
            const unsigned long long u = u0 + (unsigned long long)groups * i;
            if (u >= p.units) continue;
            const Divisor d = divisor_of(most);
            if (lane == 0) p.scale[(long long)row[i] * p.blocks + block[i]] = d.scale;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int col = (int)block[i] * BQ_BLOCK + (j * LANES + lane) * VEC;
                uint8_t q[VEC];
                quantise<T, VEC>(v[j], d, q);
                store_some<VEC>(p.q + (long long)row[i] * p.q_stride + col, q, p.k - col);
            }
        }
    }
}

// Blocks of 128 x 128, one thread block each: the values stay in registers between the maximum and the division.
template <typename T, int VEC>
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
        a[i] = load_some<T, VEC>(x + row * p.x_stride, row < p.rows ? p.k - col : 0);
    }
#pragma unroll
    for (int i = 0; i < PACKS; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) most = max_abs(most, to_f32(a[i].v[e]));
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
        float v[VEC];
        uint8_t out[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = to_f32(a[i].v[e]);
        quantise<T, VEC>(v, d, out);
        if (row < p.rows) store_some<VEC>(q + row * p.q_stride, out, p.k - col);
    }
}

template <typename T, int VEC, bool GATED> int launch_rows(BqP p, cudaStream_t stream)
{
    constexpr int PER_BLOCK = BQ_THREADS / (BQ_BLOCK / VEC < 32 ? BQ_BLOCK / VEC : 32);
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
        const unsigned blocks = std::min<unsigned>((part.units + PER_BLOCK - 1) / PER_BLOCK, 148 * 8);
        const int rc = launch_behind(block_quant_kernel<T, VEC, GATED>, blocks, dim3(BQ_THREADS), 0, 1, stream, part);
        if (rc != MOE_OVL_OK) return rc;
    }
    return MOE_OVL_OK;
}

template <typename T, int VEC> int launch_tiles(const BqP &p, int depth, cudaStream_t stream)
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
    return cudaLaunchKernelEx(&cfg, block_quant_tiles_kernel<T, VEC>, p) == cudaSuccess ? MOE_OVL_OK : MOE_OVL_ERR_CUDA;
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
        if (a->tiles) return packs ? launch_tiles<T, VEC>(p, a->depth, stream) : launch_tiles<T, 1>(p, a->depth, stream);
        if (a->gated) return packs ? launch_rows<T, VEC, true>(p, stream) : launch_rows<T, 1, true>(p, stream);
        return packs ? launch_rows<T, VEC, false>(p, stream) : launch_rows<T, 1, false>(p, stream);
    });
}
