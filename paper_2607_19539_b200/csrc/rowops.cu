// Row operators in front of and between the expert products: RMS norm of a sum with an optional 8-bit output, its
// gradient, and the gated activation with an 8-bit output (entry points in include/moe_ovl.h).
//
// All of them read each element once, need one reduction over the row, and write once: they are bound by HBM.  A row is
// held in registers between the two (NV packs of VEC elements per thread), so nothing is read twice.  The row's
// threads are one block, or one warp where the row is short (several rows per block then, and no block barrier).
#include "opcommon.cuh"

using namespace moe_ovl;

namespace {

constexpr float QUANT_MAX = 127.0f;
constexpr float QUANT_TINY = 7.8886090522101181e-31f;      // 2^-100
constexpr int NORM_PARTIALS = 592;                          // most partial rows of the weight gradient: 148 SMs x 4

// Threads a block of a kernel with so many values per thread may have: the row lives in registers.
constexpr int max_threads(int values) { return values <= 16 ? 1024 : 512; }

// Sum / largest magnitude over the threads of one row.  `buf`: 32 floats that no thread of the block still reads.
__device__ __forceinline__ float row_sum(float v, float *buf)
{
    v = warp_sum(v);
    if (blockDim.x == 32) return v;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < (int)(blockDim.x >> 5) ? buf[lane] : 0.0f);
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
    const float2 t = lane < (int)(blockDim.x >> 5) ? buf[lane] : make_float2(0.0f, 0.0f);
    s = warp_sum(t.x);
    m = warp_max(t.y);
}

// scale = most / 127 and the factor that takes a value to its 8 bits; a row of (almost) nothing gives zeros.
__device__ __forceinline__ float2 quant_scale(float most)
{
    if (most < QUANT_TINY) return make_float2(0.0f, 0.0f);
    return make_float2(most / QUANT_MAX, QUANT_MAX / most);
}
// To the nearest whole number, ties to even; a NaN gives 0.
__device__ __forceinline__ int8_t quant(float v, float inverse)
{
    const int i = __float2int_rn(v * inverse);
    return (int8_t)max(-127, min(127, i));
}

struct NormP {
    int rows, d;
    float eps;
    const void *x, *residual, *weight;
    void *residual_out, *y;
    int8_t *q;
    float *scale, *rstd;
    long long x_stride, residual_stride, residual_out_stride, y_stride, q_stride;
};

// One row per block (or warp).  The row's sum of squares and the largest |h * weight| come out of ONE reduction: rstd is
// a positive factor of the whole row, so the scale of the 8-bit output needs no second pass over the normed values.
template <typename T, typename W, int VEC, int NV>
__global__ void __launch_bounds__(max_threads(VEC *NV)) add_norm_kernel(const NormP p)
{
    __shared__ float2 buf[32];
    const int row = blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.rows) return;                  // whole warps: rows share a block only as one warp each
    const T *x = static_cast<const T *>(p.x) + row * p.x_stride;
    const T *res = p.residual ? static_cast<const T *>(p.residual) + row * p.residual_stride : nullptr;
    T *h_out = p.residual_out ? static_cast<T *>(p.residual_out) + row * p.residual_out_stride : nullptr;
    const W *w = static_cast<const W *>(p.weight);
    Pack<T, VEC> a[NV], b[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c < p.d) {
            a[i] = load_pack<T, VEC>(x + c);
            if (res) b[i] = load_pack<T, VEC>(res + c);
        }
    }
    float v[NV * VEC];                          // h, then h * weight
    float sum = 0.0f, most = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c >= p.d) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i * VEC + j] = 0.0f;
            continue;
        }
        const Pack<W, VEC> wv = load_pack<W, VEC>(w + c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            // the sum is rounded to the type it is stored in: the norm is that of the stored value
            const T h = res ? from_f32<T>(to_f32(a[i].v[j]) + to_f32(b[i].v[j])) : a[i].v[j];
            a[i].v[j] = h;
            const float hf = to_f32(h);
            sum = fmaf(hf, hf, sum);
            const float t = hf * to_f32(wv.v[j]);
            v[i * VEC + j] = t;
            most = max_nan(most, fabsf(t));
        }
        if (h_out) store_pack<T, VEC>(h_out + c, a[i]);
    }
    row_sum_max(sum, most, buf);
    const float rstd = 1.0f / sqrtf(sum / (float)p.d + p.eps);
    if (threadIdx.x == 0 && p.rstd) p.rstd[row] = rstd;
    if (p.y) {
        T *y = static_cast<T *>(p.y) + row * p.y_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c < p.d) {
                Pack<T, VEC> o;
#pragma unroll
                for (int j = 0; j < VEC; ++j) o.v[j] = from_f32<T>(v[i * VEC + j] * rstd);
                store_pack<T, VEC>(y + c, o);
            }
        }
    }
    if (p.q) {
        const float2 s = quant_scale(most * rstd);
        if (threadIdx.x == 0) p.scale[row] = s.x;
        int8_t *q = p.q + row * p.q_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c < p.d) {
                Pack<int8_t, VEC> o;
#pragma unroll
                for (int j = 0; j < VEC; ++j) o.v[j] = quant(v[i * VEC + j] * rstd, s.y);
                store_pack<int8_t, VEC>(q + c, o);
            }
        }
    }
}

struct NormBackP {
    int rows, d;
    const void *dy, *h, *weight, *d_residual;
    const float *rstd;
    void *dx;
    float *partial;                             // [gridDim.x * blockDim.y][d] sums of dy * n, or NULL
    long long dy_stride, h_stride, d_residual_stride, dx_stride;
};

// Every block (or warp) takes rows at a fixed distance and keeps its columns' share of the weight gradient in registers
// over all of them; the partial rows are added up in a fixed order by reduce_partials_kernel: no atomics, same bits.
template <typename T, typename W, int VEC, int NV>
__global__ void __launch_bounds__(max_threads(VEC *NV)) add_norm_backward_kernel(const NormBackP p)
{
    __shared__ float buf[2][32];
    float acc[NV * VEC];
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i) acc[i] = 0.0f;
    const int first = blockIdx.x * blockDim.y + threadIdx.y, step = gridDim.x * blockDim.y;
    const W *w = static_cast<const W *>(p.weight);
    int turn = 0;
    for (int row = first; row < p.rows; row += step, turn ^= 1) {
        const T *dy = static_cast<const T *>(p.dy) + row * p.dy_stride;
        const T *h = static_cast<const T *>(p.h) + row * p.h_stride;
        const T *dr = p.d_residual ? static_cast<const T *>(p.d_residual) + row * p.d_residual_stride : nullptr;
        T *dx = static_cast<T *>(p.dx) + row * p.dx_stride;
        const float rstd = p.rstd[row];
        Pack<T, VEC> a[NV], b[NV], r[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c < p.d) {
                a[i] = load_pack<T, VEC>(dy + c);
                b[i] = load_pack<T, VEC>(h + c);
                if (dr) r[i] = load_pack<T, VEC>(dr + c);
            }
        }
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c >= p.d) continue;
            const Pack<W, VEC> wv = load_pack<W, VEC>(w + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float n = to_f32(b[i].v[j]) * rstd, t = to_f32(a[i].v[j]);
                acc[i * VEC + j] = fmaf(t, n, acc[i * VEC + j]);
                dot = fmaf(t * to_f32(wv.v[j]), n, dot);
            }
        }
        const float mean = row_sum(dot, buf[turn]) / (float)p.d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c >= p.d) continue;
            const Pack<W, VEC> wv = load_pack<W, VEC>(w + c);
            Pack<T, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float n = to_f32(b[i].v[j]) * rstd, g = to_f32(a[i].v[j]) * to_f32(wv.v[j]);
                float v = rstd * (g - n * mean);
                if (dr) v += to_f32(r[i].v[j]);
                o.v[j] = from_f32<T>(v);
            }
            store_pack<T, VEC>(dx + c, o);
        }
    }
    if (!p.partial) return;
    float *out = p.partial + (long long)first * p.d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c < p.d) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) out[c + j] = acc[i * VEC + j];
        }
    }
}

// dweight[c] = sum of the partial rows, each column by 16 threads and then in one tree: a fixed order.
__global__ void __launch_bounds__(512) reduce_partials_kernel(const float *partial, int count, int d, float *dweight)
{
    __shared__ float buf[16][33];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float s = 0.0f;
    if (c < d)
        for (int i = threadIdx.y; i < count; i += 16) s += partial[(long long)i * d + c];
    buf[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    for (int o = 8; o > 0; o >>= 1) {
        if (threadIdx.y < o) buf[threadIdx.y][threadIdx.x] += buf[threadIdx.y + o][threadIdx.x];
        __syncthreads();
    }
    if (threadIdx.y == 0 && c < d) dweight[c] = buf[0][threadIdx.x];
}

struct SwigluP {
    int rows, f;
    const void *x;
    int8_t *q;
    float *scale;
    long long x_stride, q_stride;
};

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(max_threads(VEC *NV)) swiglu_quant_kernel(const SwigluP p)
{
    __shared__ float buf[32];
    const int row = blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.rows) return;
    const T *g = static_cast<const T *>(p.x) + row * p.x_stride, *u = g + p.f;
    Pack<T, VEC> a[NV], b[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c < p.f) {
            a[i] = load_pack<T, VEC>(g + c);
            b[i] = load_pack<T, VEC>(u + c);
        }
    }
    float v[NV * VEC], most = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float t = 0.0f;
            if (c < p.f) {
                const float gf = to_f32(a[i].v[j]);
                t = gf / (1.0f + expf(-gf)) * to_f32(b[i].v[j]);
            }
            v[i * VEC + j] = t;
            most = max_nan(most, fabsf(t));
        }
    }
    most = row_max(most, buf);
    const float2 s = quant_scale(most);
    if (threadIdx.x == 0) p.scale[row] = s.x;
    int8_t *q = p.q + row * p.q_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c < p.f) {
            Pack<int8_t, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) o.v[j] = quant(v[i * VEC + j], s.y);
            store_pack<int8_t, VEC>(q + c, o);
        }
    }
}

// How a row of `width` elements is spread: threads per row, packs per thread, rows per block.
struct RowShape { int threads, packs, rows_per_block; };

RowShape row_shape(int rows, int width, int vec, int want_packs)
{
    RowShape s;
    const int packs = (width + vec - 1) / vec;
    // few rows leave SMs idle whatever the block is: the latency of one row counts, so a thread takes one pack
    const int want = rows <= 296 ? 1 : want_packs;
    int nv = 1;
    while (nv < want && packs > 32 * nv) nv *= 2;
    // a pack more per thread until the block is small enough for the registers
    auto threads = [&](int n) { return ((packs + n - 1) / n + 31) / 32 * 32; };
    while (threads(nv) > max_threads(vec * nv)) nv *= 2;
    s.packs = nv;
    s.threads = threads(nv);
    s.rows_per_block = s.threads == 32 ? 4 : 1;
    return s;
}

template <int N> struct Count { static constexpr int value = N; };
// Calls f with the number of packs as a constant: 1, 2, 4 ... up to 64 / VEC values' worth.
template <int VEC, typename F> int with_packs(int packs, F f)
{
    if (packs <= 1) return f(Count<1>());
    if (packs == 2) return f(Count<2>());
    if (packs == 4) return f(Count<4>());
    if constexpr (VEC <= 8) if (packs == 8) return f(Count<8>());
    if constexpr (VEC <= 4) if (packs == 16) return f(Count<16>());
    if constexpr (VEC <= 1) if (packs == 32) return f(Count<32>());
    if constexpr (VEC <= 1) if (packs == 64) return f(Count<64>());
    return MOE_OVL_ERR_UNSUPPORTED;
}

template <typename T> constexpr int vec_of() { return 16 / (int)sizeof(T); }

bool rows_ok(const void *p, int64_t stride, int vec, int bytes) { return aligned(p, (size_t)vec * bytes) && stride % vec == 0; }

// A matrix whose rows do not overlap (or that has one row) and whose offsets stay within 63 bits.
bool stride_ok(int64_t stride, int rows, int width) { return (rows <= 1 || stride >= width) && stride >= 0 && stride < (1ll << 40); }

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
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->dtype), ws = dtype_bytes(a->weight_dtype);
    if (!a->x || !a->weight || !aligned(a->x, es) || !aligned(a->residual, es) || !aligned(a->residual_out, es) || !aligned(a->y, es) ||
        !aligned(a->weight, ws) || !aligned(a->scale, 4) || !aligned(a->rstd, 4))
        return MOE_OVL_ERR_INVALID_ARG;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    NormP p = {a->rows, a->d, a->eps, a->x, a->residual, a->weight, a->residual_out, a->y, a->q, a->scale, a->rstd,
               a->x_stride, a->residual_stride, a->residual_out_stride, a->y_stride, a->q_stride};
    const int vec = 16 / es;
    const bool wide = a->d % vec == 0 && rows_ok(a->x, a->x_stride, vec, es) && aligned(a->weight, (size_t)vec * ws) &&
                      (!a->residual || rows_ok(a->residual, a->residual_stride, vec, es)) &&
                      (!a->residual_out || rows_ok(a->residual_out, a->residual_out_stride, vec, es)) &&
                      (!a->y || rows_ok(a->y, a->y_stride, vec, es)) && (!a->q || rows_ok(a->q, a->q_stride, vec, 1));
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto w, auto v) {
            using W = decltype(w);
            constexpr int VEC = decltype(v)::value;
            const RowShape s = row_shape(p.rows, p.d, VEC, VEC == 1 ? 8 : 2);
            return with_packs<VEC>(s.packs, [&](auto n) {
                const int blocks = (p.rows + s.rows_per_block - 1) / s.rows_per_block;
                add_norm_kernel<T, W, VEC, decltype(n)::value>
                    <<<blocks, dim3(s.threads, s.rows_per_block), 0, static_cast<cudaStream_t>(a->stream)>>>(p);
                return launched();
            });
        };
        auto by_weight = [&](auto v) { return a->weight_dtype == a->dtype ? launch(T(), v) : launch(0.0f, v); };
        return wide ? by_weight(Count<vec_of<T>()>()) : by_weight(Count<1>());
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
    NormBackP p = {a->rows, a->d, a->dy, a->h, a->weight, a->d_residual, a->rstd, a->dx,
                   a->dweight ? static_cast<float *>(a->workspace) : nullptr, a->dy_stride, a->h_stride, a->d_residual_stride, a->dx_stride};
    const int vec = 16 / es;
    const bool wide = a->d % vec == 0 && rows_ok(a->dy, a->dy_stride, vec, es) && rows_ok(a->h, a->h_stride, vec, es) &&
                      rows_ok(a->dx, a->dx_stride, vec, es) && aligned(a->weight, (size_t)vec * ws) &&
                      (!a->d_residual || rows_ok(a->d_residual, a->d_residual_stride, vec, es));
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto w, auto v) {
            using W = decltype(w);
            constexpr int VEC = decltype(v)::value;
            const RowShape s = row_shape(p.rows, p.d, VEC, VEC == 1 ? 8 : 1);
            return with_packs<VEC>(s.packs, [&](auto n) {
                // rows_per_block rows at a time; at most NORM_PARTIALS partial rows in all
                int blocks = (p.rows + s.rows_per_block - 1) / s.rows_per_block;
                blocks = blocks < NORM_PARTIALS / s.rows_per_block ? blocks : NORM_PARTIALS / s.rows_per_block;
                int rows_per_block = s.rows_per_block;
                if (p.rows < rows_per_block) rows_per_block = p.rows, blocks = 1;
                if (blocks * rows_per_block > p.rows) blocks = p.rows / rows_per_block;
                add_norm_backward_kernel<T, W, VEC, decltype(n)::value>
                    <<<blocks, dim3(s.threads, rows_per_block), 0, stream>>>(p);
                if (p.partial)
                    reduce_partials_kernel<<<(p.d + 31) / 32, dim3(32, 16), 0, stream>>>(p.partial, blocks * rows_per_block, p.d, a->dweight);
                return launched();
            });
        };
        auto by_weight = [&](auto v) { return a->weight_dtype == a->dtype ? launch(T(), v) : launch(0.0f, v); };
        return wide ? by_weight(Count<vec_of<T>()>()) : by_weight(Count<1>());
    });
}

extern "C" int moe_ovl_swiglu_quant(const moe_ovl_swiglu_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->f < 1 || a->flags != 0) return MOE_OVL_ERR_INVALID_ARG;
    if (!known_dtype(a->dtype)) return MOE_OVL_ERR_INVALID_ARG;
    if (a->f > MOE_OVL_MAX_ROW) return MOE_OVL_ERR_UNSUPPORTED;
    if (!stride_ok(a->gate_up_stride, a->rows, 2 * a->f) || !stride_ok(a->q_stride, a->rows, a->f)) return MOE_OVL_ERR_INVALID_ARG;
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->dtype);
    if (!a->gate_up || !a->q || !a->scale || !aligned(a->gate_up, es) || !aligned(a->scale, 4)) return MOE_OVL_ERR_INVALID_ARG;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const SwigluP p = {a->rows, a->f, a->gate_up, a->q, a->scale, a->gate_up_stride, a->q_stride};
    const int vec = 16 / es;
    const bool wide = a->f % vec == 0 && rows_ok(a->gate_up, a->gate_up_stride, vec, es) && rows_ok(a->q, a->q_stride, vec, 1);
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto v) {
            constexpr int VEC = decltype(v)::value;
            const RowShape s = row_shape(p.rows, p.f, VEC, VEC == 1 ? 8 : 2);
            return with_packs<VEC>(s.packs, [&](auto n) {
                const int blocks = (p.rows + s.rows_per_block - 1) / s.rows_per_block;
                swiglu_quant_kernel<T, VEC, decltype(n)::value>
                    <<<blocks, dim3(s.threads, s.rows_per_block), 0, static_cast<cudaStream_t>(a->stream)>>>(p);
                return launched();
            });
        };
        return wide ? launch(Count<vec_of<T>()>()) : launch(Count<1>());
    });
}
