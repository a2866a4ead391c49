// Router of the expert layer and its gradient (moe_ovl_route, moe_ovl_route_backward in include/moe_ovl.h).
//
// One warp per row.  A lane holds NR logits in registers, V neighbours at a time, so a row is read once.  Choices are
// compared as 32-bit keys whose unsigned order is the order of the floats (0 = masked): the largest key over the warp
// is one reduction instruction, and the lowest index among the lanes that hold it is a second one, which is what makes
// ties go to the lowest index.
#include <algorithm>

#include "opcommon.cuh"

using namespace moe_ovl;

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int ROUTE_WARPS = 8;
constexpr int ROUTE_BLOCKS = 148 * 8;      // every SM full of warps

struct RouteP {
    int rows, experts, k, groups, per_group, top_groups, group_best;
    bool sigmoid, renormalise, by_score;   // by_score: choices are scores (+ bias); else the logits themselves
    float gate_scale;
    const void *logits;
    const float *bias;
    int *expert;
    float *gate;
    int *counts;
    long long stride;
};

// Unsigned keys in the order of the floats; -inf and NaN (masked) become 0, both zeros one key.
__device__ __forceinline__ unsigned key_of(float v)
{
    const unsigned u = __float_as_uint(v + 0.0f);
    return v > -INFINITY ? ((u & 0x80000000u) ? ~u : (u | 0x80000000u)) : 0u;
}
__device__ __forceinline__ float value_of(unsigned key)
{
    return __uint_as_float((key & 0x80000000u) ? (key & 0x7fffffffu) : ~key);
}
// A logit as it is used: +inf is the largest finite value, a NaN is -inf.
__device__ __forceinline__ float usable(float v) { return v != v ? -INFINITY : fminf(v, 3.402823466e+38f); }
__device__ __forceinline__ float sigmoid_of(float v) { return 1.0f / (1.0f + expf(-v)); }

// Index of a lane's r-th logit.
template <int V> __device__ __forceinline__ int expert_at(int r, int lane) { return (r / V) * (32 * V) + lane * V + r % V; }

template <typename T, int NR, int V>
__device__ __forceinline__ void load_row(const T *row, int experts, int lane, float (&l)[NR])
{
#pragma unroll
    for (int r = 0; r < NR; r += V) {
        const int e = expert_at<V>(r, lane);
        if (e < experts) {
            const Pack<T, V> a = load_pack<T, V>(row + e);
#pragma unroll
            for (int j = 0; j < V; ++j) l[r + j] = usable(to_f32(a.v[j]));
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) l[r + j] = -INFINITY;
        }
    }
}

// exp(l - m) with l = -inf giving 0 also where the whole row is masked
__device__ __forceinline__ float exp_from(float l, float m) { return l > -INFINITY ? expf(l - m) : 0.0f; }

template <typename T, int NR, int V, bool GROUPS>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_kernel(const RouteP p)
{
    extern __shared__ int histogram[];
    const int lane = threadIdx.x & 31;
    if (p.counts) {
        for (int i = threadIdx.x; i < p.experts; i += blockDim.x) histogram[i] = 0;
        __syncthreads();
    }
    int group[GROUPS ? NR : 1];
    if (GROUPS) {
#pragma unroll
        for (int r = 0; r < NR; ++r) group[r] = expert_at<V>(r, lane) / p.per_group;   // beyond the last: >= groups
    }
    for (int row = blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5); row < p.rows; row += gridDim.x * ROUTE_WARPS) {
        const T *logits = static_cast<const T *>(p.logits) + row * p.stride;
        float l[NR];
        load_row<T, NR, V>(logits, p.experts, lane, l);
        float top = -INFINITY, total = 0.0f;            // softmax over the row
        if (!p.sigmoid && (p.by_score || !p.renormalise)) {
#pragma unroll
            for (int r = 0; r < NR; ++r) top = fmaxf(top, l[r]);
            top = warp_max(top);
#pragma unroll
            for (int r = 0; r < NR; ++r) total += exp_from(l[r], top);
            total = warp_sum(total);
        }
        unsigned key[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float c = l[r];
            if (p.by_score && c > -INFINITY) {
                const int e = expert_at<V>(r, lane);
                c = p.sigmoid ? sigmoid_of(c) : expf(c - top) / total;
                if (p.bias) c += p.bias[e];
            }
            key[r] = key_of(c);
        }
        if (GROUPS) {
            float mine = -INFINITY;                     // value of group `lane`
            for (int g = 0; g < p.groups; ++g) {
                unsigned first = 0, second = 0;
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    const unsigned x = group[r] == g ? key[r] : 0u;
                    second = max(second, min(first, x));
                    first = max(first, x);
                }
                const unsigned best = __reduce_max_sync(FULL, first);
                float v = best ? value_of(best) : -INFINITY;
                if (p.group_best == 2) {
                    const int owner = __ffs(__ballot_sync(FULL, first == best)) - 1;
                    const unsigned next = __reduce_max_sync(FULL, lane == owner ? second : first);
                    if (next) v += value_of(next);
                }
                if (lane == g) mine = v;
            }
            int before = 0;                             // groups that come first: larger, or equal with a lower index
            for (int g = 0; g < p.groups; ++g) {
                const float v = __shfl_sync(FULL, mine, g);
                before += v > mine || (v == mine && g < lane);
            }
            const unsigned taken = __ballot_sync(FULL, lane < p.groups && before < p.top_groups);
#pragma unroll
            for (int r = 0; r < NR; ++r)
                if (group[r] >= 32 || !(taken >> group[r] & 1u)) key[r] = 0;
        }
        int chosen = -1;                                // of slot `lane`
        for (int j = 0; j < p.k; ++j) {
            unsigned best = 0;
#pragma unroll
            for (int r = 0; r < NR; ++r) best = max(best, key[r]);
            best = __reduce_max_sync(FULL, best);
            if (best == 0) break;                       // uniform: nothing is left
            unsigned at = 0xffffffffu;
#pragma unroll
            for (int r = NR - 1; r >= 0; --r)
                if (key[r] == best) at = expert_at<V>(r, lane);
            at = __reduce_min_sync(FULL, at);
#pragma unroll
            for (int r = 0; r < NR; ++r)
                if (expert_at<V>(r, lane) == (int)at) key[r] = 0;
            if (lane == j) chosen = (int)at;
        }
        const float x = chosen >= 0 ? usable(to_f32(logits[chosen])) : -INFINITY;
        float g = 0.0f;
        if (p.sigmoid) {
            g = chosen >= 0 ? sigmoid_of(x) : 0.0f;
        } else if (p.renormalise) {
            g = exp_from(x, warp_max(x));
        } else {
            g = exp_from(x, top) / total;
        }
        if (p.renormalise) {
            const float sum = warp_sum(g);
            g = sum > 0.0f ? g / sum : 0.0f;
        }
        if (lane < p.k) {
            p.expert[(long long)row * p.k + lane] = chosen;
            p.gate[(long long)row * p.k + lane] = chosen >= 0 ? p.gate_scale * g : 0.0f;
            if (p.counts && chosen >= 0) atomicAdd(&histogram[chosen], 1);
        }
    }
    if (p.counts) {
        __syncthreads();
        for (int i = threadIdx.x; i < p.experts; i += blockDim.x) {
            if (gridDim.x == 1) p.counts[i] = histogram[i];
            else if (histogram[i]) atomicAdd(&p.counts[i], histogram[i]);      // whole numbers: any order
        }
    }
}

struct RouteBackP {
    int rows, experts, k;
    bool sigmoid, renormalise;
    float gate_scale;
    const void *logits;
    const int *expert;
    const float *dgate;
    void *dlogits;
    long long stride, out_stride;
};

// dlogits of one row: with s the scores, c = gate_scale and, over the chosen, w = s / sum(s):
//   softmax              s_i (c dgate_i - sum c dgate s)     every expert (dgate 0 where not chosen)
//   softmax, renormalised w_j (c dgate_j - sum c dgate w)    the chosen ones, 0 elsewhere
//   sigmoid              c dgate_j s_j (1 - s_j)
//   sigmoid, renormalised w_j (1 - s_j) (c dgate_j - sum c dgate w)
template <typename T, int NR, int V>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_backward_kernel(const RouteBackP p)
{
    const int lane = threadIdx.x & 31;
    for (int row = blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5); row < p.rows; row += gridDim.x * ROUTE_WARPS) {
        const T *logits = static_cast<const T *>(p.logits) + row * p.stride;
        T *out = static_cast<T *>(p.dlogits) + row * p.out_stride;
        int e = -1;
        float d = 0.0f;
        if (lane < p.k) {
            e = p.expert[(long long)row * p.k + lane];
            d = p.gate_scale * p.dgate[(long long)row * p.k + lane];
            if (e < 0 || e >= p.experts) e = -1, d = 0.0f;
        }
        float x = e >= 0 ? usable(to_f32(logits[e])) : -INFINITY;
        if (!(x > -INFINITY)) d = 0.0f;
        float dense[NR];                                // what an expert that was not chosen gets
#pragma unroll
        for (int r = 0; r < NR; ++r) dense[r] = 0.0f;
        float mine;
        if (!p.sigmoid && !p.renormalise) {
            float l[NR];
            load_row<T, NR, V>(logits, p.experts, lane, l);
            float top = -INFINITY, total = 0.0f;
#pragma unroll
            for (int r = 0; r < NR; ++r) top = fmaxf(top, l[r]);
            top = warp_max(top);
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                dense[r] = exp_from(l[r], top);
                total += dense[r];
            }
            total = warp_sum(total);
            const float inv = total > 0.0f ? 1.0f / total : 0.0f;
            const float s = exp_from(x, top) * inv;
            const float dot = warp_sum(d * s);
#pragma unroll
            for (int r = 0; r < NR; ++r) dense[r] *= -inv * dot;
            mine = s * (d - dot);
        } else {
            const float s = p.sigmoid ? (x > -INFINITY ? sigmoid_of(x) : 0.0f) : exp_from(x, warp_max(x));
            float w = s, dot = 0.0f;
            if (p.renormalise) {
                const float sum = warp_sum(s);
                w = sum > 0.0f ? s / sum : 0.0f;
                dot = warp_sum(d * w);
            }
            mine = w * (d - dot) * (p.sigmoid ? 1.0f - s : 1.0f);
        }
        __syncwarp();                                   // every logit of the row has been read: out may be logits
#pragma unroll
        for (int r = 0; r < NR; r += V) {
            const int at = expert_at<V>(r, lane);
            if (at < p.experts) {
                Pack<T, V> o;
#pragma unroll
                for (int j = 0; j < V; ++j) o.v[j] = from_f32<T>(dense[r + j]);
                store_pack<T, V>(out + at, o);
            }
        }
        __syncwarp();                                   // the chosen ones' values come after the others'
        if (e >= 0) out[e] = from_f32<T>(mine);
    }
}

template <int A, int B> struct Pair { static constexpr int nr = A, v = B; };
// Calls f with the logits per lane and, where rows allow it, as many neighbours as 16 bytes hold.
template <typename T, typename F> int with_row(int experts, bool wide, F f)
{
    constexpr int W = 16 / (int)sizeof(T);
    if (experts <= 32) return f(Pair<1, 1>());
    if (experts <= 64) return wide ? f(Pair<2, 2>()) : f(Pair<2, 1>());
    if (experts <= 128) return wide ? f(Pair<4, 4>()) : f(Pair<4, 1>());
    if (experts <= 256) return wide ? f(Pair<8, W>()) : f(Pair<8, 1>());
    if (experts <= 512) return wide ? f(Pair<16, W>()) : f(Pair<16, 1>());
    return wide ? f(Pair<32, W>()) : f(Pair<32, 1>());
}
// Neighbours per load that with_row takes for a wide row.
template <typename T> int wide_of(int experts)
{
    const int w = 16 / (int)sizeof(T);
    return experts <= 32 ? 1 : experts <= 64 ? 2 : experts <= 128 ? std::min(4, w) : w;
}

int blocks_for(int rows) { return std::min((rows + ROUTE_WARPS - 1) / ROUTE_WARPS, ROUTE_BLOCKS); }

}  // namespace

extern "C" int moe_ovl_route(const moe_ovl_route_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->num_experts < 1 || a->top_k < 1 ||
        a->top_k > a->num_experts || !known_dtype(a->dtype) || (a->score != MOE_OVL_SCORE_SOFTMAX && a->score != MOE_OVL_SCORE_SIGMOID) ||
        a->num_groups < 1 || a->num_experts % a->num_groups != 0 || a->top_groups < 1 || a->top_groups > a->num_groups ||
        (a->group_best != 1 && a->group_best != 2) || (a->renormalise != 0 && a->renormalise != 1) || !(a->gate_scale == a->gate_scale))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->num_experts > MOE_OVL_MAX_ROUTED || a->top_k > MOE_OVL_MAX_TOP_K || a->num_groups > 32) return MOE_OVL_ERR_UNSUPPORTED;
    const int es = dtype_bytes(a->dtype);
    if (a->rows > 0 && (!a->logits || !a->expert || !a->gate || !aligned(a->logits, es) || !aligned(a->expert, 4) || !aligned(a->gate, 4) ||
                        a->logits_stride >= (1ll << 40) || (a->rows > 1 && a->logits_stride < a->num_experts)))
        return MOE_OVL_ERR_INVALID_ARG;
    if (!aligned(a->bias, 4) || !aligned(a->counts, 4)) return MOE_OVL_ERR_INVALID_ARG;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    const int blocks = blocks_for(a->rows);
    // one block stores its counts; several add to them
    if (a->counts && blocks != 1 && cudaMemsetAsync(a->counts, 0, (size_t)a->num_experts * 4, stream) != cudaSuccess) return MOE_OVL_ERR_CUDA;
    if (a->rows == 0) return MOE_OVL_OK;
    RouteP p = {a->rows, a->num_experts, a->top_k, a->num_groups, a->num_experts / a->num_groups, a->top_groups, a->group_best,
                a->score == MOE_OVL_SCORE_SIGMOID, a->renormalise != 0, a->bias != nullptr || (a->num_groups > 1 && a->group_best == 2),
                a->gate_scale, a->logits, a->bias, a->expert, a->gate, a->counts, a->logits_stride};
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        const int v = wide_of<T>(p.experts);
        const bool wide = p.experts % v == 0 && p.stride % v == 0 && aligned(p.logits, v * sizeof(T));
        return with_row<T>(p.experts, wide, [&](auto c) {
            constexpr int NR = decltype(c)::nr, V = std::min(decltype(c)::v, 16 / (int)sizeof(T));
            const size_t smem = p.counts ? (size_t)p.experts * 4 : 0;
            if (p.groups > 1) route_kernel<T, NR, V, true><<<blocks, 32 * ROUTE_WARPS, smem, stream>>>(p);
            else route_kernel<T, NR, V, false><<<blocks, 32 * ROUTE_WARPS, smem, stream>>>(p);
            return launched();
        });
    });
}

extern "C" int moe_ovl_route_backward(const moe_ovl_route_backward_args *a)
{
    if (!a || a->struct_size != sizeof(*a) || a->device < 0 || a->rows < 0 || a->num_experts < 1 || a->top_k < 1 ||
        a->top_k > a->num_experts || !known_dtype(a->dtype) || (a->score != MOE_OVL_SCORE_SOFTMAX && a->score != MOE_OVL_SCORE_SIGMOID) ||
        (a->renormalise != 0 && a->renormalise != 1) || a->flags != 0 || !(a->gate_scale == a->gate_scale))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->num_experts > MOE_OVL_MAX_ROUTED || a->top_k > MOE_OVL_MAX_TOP_K) return MOE_OVL_ERR_UNSUPPORTED;
    if (a->rows == 0) return MOE_OVL_OK;
    const int es = dtype_bytes(a->dtype);
    if (!a->logits || !a->expert || !a->dgate || !a->dlogits || !aligned(a->logits, es) || !aligned(a->dlogits, es) || !aligned(a->expert, 4) ||
        !aligned(a->dgate, 4) || a->logits_stride >= (1ll << 40) || a->dlogits_stride >= (1ll << 40) ||
        (a->rows > 1 && (a->logits_stride < a->num_experts || a->dlogits_stride < a->num_experts)))
        return MOE_OVL_ERR_INVALID_ARG;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    RouteBackP p = {a->rows, a->num_experts, a->top_k, a->score == MOE_OVL_SCORE_SIGMOID, a->renormalise != 0, a->gate_scale,
                    a->logits, a->expert, a->dgate, a->dlogits, a->logits_stride, a->dlogits_stride};
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        const int v = wide_of<T>(p.experts);
        const bool wide = p.experts % v == 0 && p.stride % v == 0 && p.out_stride % v == 0 && aligned(p.logits, v * sizeof(T)) &&
                          aligned(p.dlogits, v * sizeof(T));
        return with_row<T>(p.experts, wide, [&](auto c) {
            constexpr int NR = decltype(c)::nr, V = std::min(decltype(c)::v, 16 / (int)sizeof(T));
            route_backward_kernel<T, NR, V><<<blocks_for(p.rows), 32 * ROUTE_WARPS, 0, static_cast<cudaStream_t>(a->stream)>>>(p);
            return launched();
        });
    });
}
