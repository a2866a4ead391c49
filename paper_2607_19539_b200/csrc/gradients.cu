// Norm of a list of gradients and clipping by it (moe_ovl_grad_norm, moe_ovl_clip_grads in include/moe_ovl.h).
//
// A list goes to the kernel as a parameter, up to LIST_LONG tensors per launch, so no table has to be copied or kept on the device.  The
// elements of all its tensors are dealt out in chunks, a contiguous run of them to each block, which finds its first tensor by bisection
// and walks on from there.  Squares are summed in 32 bits over a thread's share of a chunk (64 values at most, two sums of 32) and in 64 bits beyond; a share whose 32-bit
// sum overflows, is not a number, or is so small that squares may have vanished, is summed again in 64, over the same values.  Every block's sum has its place in the workspace (or, of a small
// list, in its shared memory) and one block adds them up in order: the same call gives the same bits.
#include <algorithm>

#include "opcommon.cuh"
#include "ptx.cuh"

using namespace moe_ovl;

namespace {

constexpr int GN_THREADS = 256, GN_PER_THREAD = 64, GN_CHUNK = GN_THREADS * GN_PER_THREAD;
constexpr int GN_BLOCKS = 148 * 8;           // most blocks of a launch
constexpr int LIST_SHORT = 32, LIST_LONG = 960;      // 32 KB of parameters are allowed

struct Tensor {
    const void *from;
    void *to;
    long long size;
    unsigned chunk;                          // chunks in front of it
    int dtype;
};
template <int N> struct TensorList {
    int count;
    unsigned chunks;
    Tensor t[N];
};

template <int N> __device__ __forceinline__ int tensor_at(const TensorList<N> &list, unsigned chunk)
{
    int lo = 0, hi = list.count - 1;         // the last one whose first chunk is not behind
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (list.t[mid].chunk <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// The values of a chunk that are this thread's: packs(index of the first value of up to AT_ONCE packs, GN_THREADS packs apart, how many), whose loads come before anything is done with them, and one(index) for
// values in front of the first pack of 16 bytes and behind the last.
template <int VEC, int AT_ONCE, typename Packs, typename One>
__device__ __forceinline__ void for_values(long long begin, long long end, int head, Packs packs, One one)
{
    const long long first = min(begin + head, end), count = (end - first) / VEC;
    if (begin + (int)threadIdx.x < first) one(begin + (int)threadIdx.x);
    for (long long i = threadIdx.x; i < count; i += AT_ONCE * GN_THREADS) {
        const int n = (int)min((count - i + GN_THREADS - 1) / GN_THREADS, (long long)AT_ONCE);
        packs(first + i * VEC, n);
    }
    const long long last = first + count * VEC + (int)threadIdx.x;
    if (last < end) one(last);
}
template <typename F> __device__ __forceinline__ void for_each(long long begin, long long end, F f)
{
    for (long long i = begin + (int)threadIdx.x; i < end; i += GN_THREADS) f(i);
}
template <typename T, int AT_ONCE> struct Packs { Pack<T, 16 / sizeof(T)> pack[AT_ONCE]; };
template <int AT_ONCE, typename T> __device__ __forceinline__ Packs<T, AT_ONCE> load_packs(const T *p, int n)
{
    constexpr int VEC = 16 / sizeof(T);
    Packs<T, AT_ONCE> r;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
        if (k < n) r.pack[k] = load_pack<T, VEC>(p + k * GN_THREADS * VEC);
        else *reinterpret_cast<uint4 *>(&r.pack[k]) = make_uint4(0, 0, 0, 0);
    }
    return r;
}
template <typename T> __device__ __forceinline__ int head_of(const T *p) { return (int)((16u - ((unsigned)(unsigned long long)p & 15u)) & 15u) / (int)sizeof(T); }

template <typename T> __device__ __forceinline__ double chunk_sum(const T *x, long long begin, long long end)
{
    constexpr int VEC = 16 / sizeof(T);
    const int head = head_of(x + begin);
    float2 sum = make_float2(0.0f, 0.0f);
    unsigned bits = 0;                       // of anything but zeros, of either sign
    constexpr unsigned UNSIGNED = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    constexpr int AT_ONCE = 4;               // 8: 146 us instead of 121 for 0.84 GB
    for_values<VEC, AT_ONCE>(begin, end, head, [&](long long i, int n) {
        const Packs<T, AT_ONCE> a = load_packs<AT_ONCE>(x + i, n);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const uint4 raw = *reinterpret_cast<const uint4 *>(&a.pack[k]);
            bits |= (raw.x | raw.y | raw.z | raw.w) & UNSIGNED;
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const float2 v = to_f32x2(&a.pack[k].v[e]);
                sum = fma2(v, v, sum);
            }
        }
    }, [&](long long i) {
        const float v = to_f32(x[i]);
        sum.x = fmaf(v, v, sum.x);
        bits |= __float_as_uint(v) & 0x7fffffffu;
    });
    const float both_sums = sum.x + sum.y;
    if (both_sums >= 1e-30f && both_sums <= 1e38f) return (double)both_sums;
    if (bits == 0) return 0.0;
    // the same values once more: each thread decides for itself, so its second sum has to be over its own share
    double wide = 0.0;
    auto add = [&](float v) { wide += (double)v * (double)v; };
    for_values<VEC, 1>(begin, end, head, [&](long long i, int) {
        const Pack<T, VEC> a = load_pack<T, VEC>(x + i);
#pragma unroll
        for (int e = 0; e < VEC; ++e) add(to_f32(a.v[e]));
    }, [&](long long i) { add(to_f32(x[i])); });
    return wide;
}

__device__ __forceinline__ double block_sum(double v, double *s)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threadIdx.x % 32 == 0) s[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0;
    for (unsigned i = 0; i < blockDim.x / 32; ++i) v += s[i];
    return v;
}

// The squares of this block's run of chunks, in every thread.
template <int N> __device__ __forceinline__ double run_sum(const TensorList<N> &list, double *s)
{
    const unsigned first = (unsigned)((unsigned long long)list.chunks * blockIdx.x / gridDim.x);
    const unsigned last = (unsigned)((unsigned long long)list.chunks * (blockIdx.x + 1) / gridDim.x);
    double sum = 0.0;
    int at = first < last ? tensor_at(list, first) : 0;
    for (unsigned c = first; c < last; ++c) {
        while (at + 1 < list.count && list.t[at + 1].chunk <= c) ++at;
        const Tensor &t = list.t[at];
        const long long begin = (long long)(c - t.chunk) * GN_CHUNK, end = min(begin + GN_CHUNK, t.size);
        if (t.dtype == MOE_OVL_BF16) sum += chunk_sum(static_cast<const __nv_bfloat16 *>(t.from), begin, end);
        else if (t.dtype == MOE_OVL_F16) sum += chunk_sum(static_cast<const __half *>(t.from), begin, end);
        else sum += chunk_sum(static_cast<const float *>(t.from), begin, end);
    }
    return block_sum(sum, s);
}

// Bound by HBM (0.84 GB in 60 tensors, bf16 or f32: 121 us, 6.9 TB/s).
template <int N>
__global__ void __launch_bounds__(GN_THREADS)
grad_norm_kernel(const __grid_constant__ TensorList<N> list, double *partial)
{
    __shared__ double s_sums[GN_THREADS / 32];
    after_previous();
    may_follow();
    const double sum = run_sum(list, s_sums);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// Small lists: one cluster, whose first block adds up the blocks' sums: one launch less, 1.7 us of the caller's time.  Bound by latency: 3.9 us on the device for
// eight chunks and 4.3 in two kernels, 5.7 and 4.7 for ten, whose blocks take two in a row, less than the caller's time that they save (in a captured step two kernels would be the faster); with 24 the second kernel is the better one in every respect.
constexpr int GN_CLUSTER = 8, GN_SMALL = 16;         // blocks; most chunks
template <int N>
__global__ void __launch_bounds__(GN_THREADS)
grad_norm_small_kernel(const __grid_constant__ TensorList<N> list, float *norm)
{
    __shared__ double s_sums[GN_THREADS / 32];
    __shared__ double s_block;
    after_previous();
    may_follow();
    const double sum = run_sum(list, s_sums);
    if (threadIdx.x == 0) s_block = sum;
    __syncwarp();
    cluster_sync_all();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        double part[GN_CLUSTER], total = 0.0;
#pragma unroll
        for (int i = 0; i < GN_CLUSTER; ++i) asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(part[i]) : "r"(map_to_cta(smem_u32(&s_block), (uint32_t)i)) : "memory");
#pragma unroll
        for (int i = 0; i < GN_CLUSTER; ++i) total += part[i];
        *norm = (float)sqrt(total);
    }
    __syncwarp();
    cluster_sync_all();                      // the sums stay until they have been read
}

constexpr int GN_FINISH = 512;
__global__ void __launch_bounds__(GN_FINISH)
grad_norm_finish_kernel(const double *partial, int count, float *norm)
{
    __shared__ double s_sums[GN_FINISH / 32];
    after_previous();
    may_follow();
    double sum = 0.0;
    for (int i = threadIdx.x; i < count; i += GN_FINISH) sum += partial[i];
    sum = block_sum(sum, s_sums);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

template <typename T> __device__ __forceinline__ void scale_chunk(const T *x, T *y, long long begin, long long end, float factor)
{
    constexpr int VEC = 16 / sizeof(T);
    auto one = [&](long long i) { y[i] = from_f32<T>(to_f32(x[i]) * factor); };
    const int head = head_of(x + begin);
    if (head != head_of(y + begin)) return for_each(begin, end, one);
    constexpr int AT_ONCE = 8;               // 4: 289 us instead of 273 for 0.84 GB
    for_values<VEC, AT_ONCE>(begin, end, head, [&](long long i, int n) {
        Packs<T, AT_ONCE> a = load_packs<AT_ONCE>(x + i, n);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) a.pack[k].v[e] = from_f32<T>(to_f32(a.pack[k].v[e]) * factor);
            if (k < n) store_pack(y + i + k * GN_THREADS * VEC, a.pack[k]);
        }
    }, one);
}

// Chunks from the last to the first: what the norm has read last is still in L2.  Bound by HBM (0.84 GB read and written: 273 us, 6.2 TB/s; norm and clipping of 0.83 GB one after the other 406-414 us).
template <int N>
__global__ void __launch_bounds__(GN_THREADS)
clip_grads_kernel(const __grid_constant__ TensorList<N> list, const float *norm, float max_norm, float eps, bool in_place)
{
    after_previous();
    may_follow();
    const float whole = *norm + eps, ratio = __fdiv_rn(max_norm, whole);
    const float factor = isinf(whole) ? 0.0f : ratio >= 1.0f || whole == 0.0f ? 1.0f : ratio;        // infinity by infinity too; NaN stays
    if (in_place && factor == 1.0f) return;
    const unsigned first = (unsigned)((unsigned long long)list.chunks * blockIdx.x / gridDim.x);
    const unsigned last = (unsigned)((unsigned long long)list.chunks * (blockIdx.x + 1) / gridDim.x);
    int at = first < last ? tensor_at(list, last - 1) : 0;
    for (unsigned c = last; c-- > first;) {
        while (list.t[at].chunk > c) --at;
        const Tensor &t = list.t[at];
        const long long begin = (long long)(c - t.chunk) * GN_CHUNK, end = min(begin + GN_CHUNK, t.size);
        if (t.dtype == MOE_OVL_BF16) scale_chunk(static_cast<const __nv_bfloat16 *>(t.from), static_cast<__nv_bfloat16 *>(t.to), begin, end, factor);
        else if (t.dtype == MOE_OVL_F16) scale_chunk(static_cast<const __half *>(t.from), static_cast<__half *>(t.to), begin, end, factor);
        else scale_chunk(static_cast<const float *>(t.from), static_cast<float *>(t.to), begin, end, factor);
    }
}

bool valid(const moe_ovl_grads_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->num_tensors < 0 || a->flags != 0 || !a->norm || !aligned(a->norm, 4)) return false;
    if (a->num_tensors > 0 && (!a->grads || !a->sizes || !a->dtypes)) return false;
    for (int i = 0; i < a->num_tensors; ++i)
        if (!known_dtype(a->dtypes[i]) || a->sizes[i] < 0 || (a->sizes[i] > 0 && (!a->grads[i] || !aligned(a->grads[i], dtype_bytes(a->dtypes[i]))))) return false;
    return true;
}
bool supported(const moe_ovl_grads_args *a)
{
    // chunks are counted in 32 bits
    long long chunks = 0;
    for (int i = 0; i < a->num_tensors; ++i) {
        if (a->sizes[i] > 1ll << 42) return false;
        chunks += (a->sizes[i] + GN_CHUNK - 1) / GN_CHUNK;
        if (chunks > 0x7fffffff) return false;
    }
    return a->num_tensors <= MOE_OVL_MAX_TENSORS;
}

// Takes the next tensors that are not empty into a list; `next` moves on.
template <int N> bool fill(TensorList<N> &list, const moe_ovl_grads_args *a, int &next)
{
    list.count = 0, list.chunks = 0;
    for (; next < a->num_tensors && list.count < N; ++next) {
        if (a->sizes[next] == 0) continue;
        list.t[list.count++] = {a->grads[next], a->out ? a->out[next] : const_cast<void *>(a->grads[next]), a->sizes[next], list.chunks, a->dtypes[next]};
        list.chunks += (unsigned)((a->sizes[next] + GN_CHUNK - 1) / GN_CHUNK);
    }
    return list.count > 0;
}
// Calls f with one list after the other; a short call's list is short, as its parameters are copied for every launch.
template <typename F> int for_lists(const moe_ovl_grads_args *a, F f)
{
    int next = 0, rc = MOE_OVL_OK;
    auto all = [&](auto &list) {
        while (rc == MOE_OVL_OK && fill(list, a, next)) rc = f(list);
    };
    if (a->num_tensors <= LIST_SHORT) {
        TensorList<LIST_SHORT> list;
        all(list);
    } else {
        TensorList<LIST_LONG> list;
        all(list);
    }
    return rc;
}
int launches_of(int num_tensors) { return (num_tensors + LIST_LONG - 1) / LIST_LONG; }

}  // namespace

extern "C" int moe_ovl_grad_norm_workspace_bytes(int32_t num_tensors, size_t *bytes)
{
    if (!bytes || num_tensors < 0) return MOE_OVL_ERR_INVALID_ARG;
    if (num_tensors > MOE_OVL_MAX_TENSORS) return MOE_OVL_ERR_UNSUPPORTED;
    *bytes = sizeof(double) * GN_BLOCKS * (size_t)std::max(launches_of(num_tensors), 1);
    return MOE_OVL_OK;
}

extern "C" int moe_ovl_grad_norm(const moe_ovl_grads_args *a)
{
    if (!valid(a)) return MOE_OVL_ERR_INVALID_ARG;
    if (!supported(a)) return MOE_OVL_ERR_UNSUPPORTED;
    size_t need = 0;
    moe_ovl_grad_norm_workspace_bytes(a->num_tensors, &need);
    if (!a->workspace || a->workspace_bytes < need || !aligned(a->workspace, 8)) return MOE_OVL_ERR_WORKSPACE;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    double *partial = static_cast<double *>(a->workspace);
    int count = 0;
    bool done = false;
    const int rc = for_lists(a, [&](auto &list) {
        constexpr int N = (int)(sizeof(list.t) / sizeof(list.t[0]));
        if (list.chunks <= GN_SMALL && a->num_tensors <= N) {
            done = true;
            return launch_behind(grad_norm_small_kernel<N>, GN_CLUSTER, dim3(GN_THREADS), 0, GN_CLUSTER, stream, list, a->norm);
        }
        const unsigned blocks = std::min<unsigned>(list.chunks, GN_BLOCKS);
        double *to = partial + count;
        count += (int)blocks;
        return launch_behind(grad_norm_kernel<N>, blocks, dim3(GN_THREADS), 0, 1, stream, list, to);
    });
    if (rc != MOE_OVL_OK || done) return rc;
    return launch_behind(grad_norm_finish_kernel, 1, dim3(GN_FINISH), 0, 1, stream, static_cast<const double *>(partial), count, a->norm);
}

extern "C" int moe_ovl_clip_grads(const moe_ovl_grads_args *a)
{
    if (!valid(a) || !(a->max_norm >= 0.0f) || !(a->eps >= 0.0f)) return MOE_OVL_ERR_INVALID_ARG;
    for (int i = 0; a->out && i < a->num_tensors; ++i)
        if (a->sizes[i] > 0 && (!a->out[i] || !aligned(a->out[i], dtype_bytes(a->dtypes[i])))) return MOE_OVL_ERR_INVALID_ARG;
    if (!supported(a)) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    return for_lists(a, [&](auto &list) {
        constexpr int N = (int)(sizeof(list.t) / sizeof(list.t[0]));
        const unsigned blocks = std::min<unsigned>(list.chunks, GN_BLOCKS);
        return launch_behind(clip_grads_kernel<N>, blocks, dim3(GN_THREADS), 0, 1, stream, list, static_cast<const float *>(a->norm), a->max_norm, a->eps,
                             a->out == nullptr);
    });
}
