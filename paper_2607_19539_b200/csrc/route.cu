// Router of the expert layer and its gradient (moe_ovl_route, moe_ovl_route_backward in include/moe_ovl.h).
//
// G lanes share a row, NR neighbouring logits each (8 up to 256 experts), so a warp works on 32 / G rows at once and what it does
// once per row -- the reductions, the rounds of the choice -- is shared by all of them.  Choices are compared as 32-bit keys whose
// unsigned order is that of the floats (0 = masked).  Every lane sorts its keys once, stably; a round then is the largest head
// over the G lanes, the first lane that holds it (its experts are the lowest: ties go to the lowest index), and a shift
// of that lane's list.  Where the logits themselves are compared and have 16 bits, a key holds the expert too, in its lower half
// and descending, so that the largest key alone is the round's answer.  Bound by instructions: at 65521 x 64, bf16, 6 chosen, a warp per
// row with a search through its keys in every round takes 45 us, G lanes with sorted lists 22 us, with the expert in the key
// 16.5 us, with the counts cleared by a kernel that lets this one in early, not by a memset, 15.0 us, of which 8.6 us are issue (594
// instructions for a warp's four rows) and the rest the order of a round's steps and the next rows' loads.
#include <algorithm>
#include <type_traits>

#include "opcommon.cuh"
#include "ptx.cuh"

using namespace moe_ovl;

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int ROUTE_THREADS = 256;
constexpr int ROUTE_BLOCKS = 148 * 4;      // what the registers allow; more of them only add counts to add up

struct RouteP {
    int rows, experts, k, groups, per_group, top_groups, group_best;
    bool sigmoid, renormalise, by_score;   // by_score: choices are scores (+ bias); else the logits themselves
    bool cluster;                          // the whole grid is one cluster, whose first block writes the counts
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
// exp(l - m) with l = -inf giving 0 also where the whole row is masked
__device__ __forceinline__ float exp_from(float l, float m) { return l > -INFINITY ? expf(l - m) : 0.0f; }

// Over the G lanes of a row.
template <int G> __device__ __forceinline__ unsigned group_max(unsigned v)
{
    if constexpr (G == 32) {
        v = __reduce_max_sync(FULL, v);
    } else {
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(FULL, v, o));
    }
    return v;
}
template <int G> __device__ __forceinline__ float group_max(float v)
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
    return v;
}
template <int G> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

// NR neighbouring logits from expert e0 on, V at a time; what lies beyond the last expert is masked.
template <typename T, int NR, int V>
__device__ __forceinline__ void load_logits(const T *row, int experts, int e0, T (&l)[NR])
{
#pragma unroll
    for (int r = 0; r < NR; r += V) {
        if (e0 + r < experts) {
            const Pack<T, V> a = load_pack<T, V>(row + e0 + r);
#pragma unroll
            for (int j = 0; j < V; ++j) l[r + j] = a.v[j];
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) l[r + j] = from_f32<T>(-INFINITY);
        }
    }
}

// Keys of 16-bit logits: the logit's order above, the expert below, so that of two equal logits the earlier has the larger key.
__device__ __forceinline__ unsigned bits_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
__device__ __forceinline__ unsigned bits_of(__half v) { return __half_as_ushort(v); }
template <typename T> __device__ __forceinline__ T from_bits(unsigned u)
{
    if constexpr (std::is_same<T, __nv_bfloat16>::value) return __ushort_as_bfloat16((unsigned short)u);
    else if constexpr (std::is_same<T, __half>::value) return __ushort_as_half((unsigned short)u);
    else return 0.0f;
}
template <typename T> __device__ __forceinline__ unsigned packed_key(T v, int e)
{
    constexpr unsigned INF = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
    unsigned u = bits_of(v);
    const bool masked = (u & 0x7fffu) > INF || u == (0x8000u | INF);
    u = u == 0x8000u ? 0u : u;                              // both zeros are one
    u = (u & 0x8000u) ? ~u : u | 0x8000u;
    return masked ? 0u : (u << 16) | (unsigned)(0xffff - e);
}
template <typename T> __device__ __forceinline__ float packed_value(unsigned key)
{
    const unsigned u = key >> 16;
    return usable(to_f32(from_bits<T>((u & 0x8000u) ? u & 0x7fffu : ~u & 0xffffu)));
}
__device__ __forceinline__ int packed_expert(unsigned key) { return 0xffff - (int)(key & 0xffffu); }

// Eight keys in descending order, none equal to another but masked ones: 19 exchanges.
__device__ __forceinline__ void sort_eight(unsigned (&k)[8])
{
    auto order = [&](int a, int b) {
        const unsigned x = max(k[a], k[b]), y = min(k[a], k[b]);
        k[a] = x, k[b] = y;
    };
    order(0, 2), order(1, 3), order(4, 6), order(5, 7);
    order(0, 4), order(1, 5), order(2, 6), order(3, 7);
    order(0, 1), order(2, 3), order(4, 5), order(6, 7);
    order(2, 4), order(3, 5);
    order(1, 4), order(3, 6);
    order(1, 2), order(3, 4), order(5, 6);
}

// Masks the keys of the experts outside the row's best groups.
template <int G, int NR>
__device__ __forceinline__ void keep_groups(const RouteP &p, unsigned (&key)[NR], int lane)
{
    const int at = lane & (G - 1), base = lane & ~(G - 1), e0 = at * NR;
    const int lanes = p.per_group / NR;                 // per group, where each holds one group's experts only
    if (p.per_group % NR == 0 && (lanes & (lanes - 1)) == 0) {
        unsigned first = 0, second = 0;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            second = max(second, min(first, key[r]));
            first = max(first, key[r]);
        }
        for (int o = 1; o < lanes; o <<= 1) {
            const unsigned f = __shfl_xor_sync(FULL, first, o), s = __shfl_xor_sync(FULL, second, o);
            second = max(min(first, f), max(second, s));
            first = max(first, f);
        }
        float mine = first ? value_of(first) : -INFINITY;
        if (p.group_best == 2 && second) mine += value_of(second);
        const int group = at / lanes;
        int before = 0;                                 // groups that come first: larger, or equal with a lower index
        for (int g = 0; g < p.groups; ++g) {
            const float v = __shfl_sync(FULL, mine, base + g * lanes);
            before += v > mine || (v == mine && g < group);
        }
        if (before >= p.top_groups) {
#pragma unroll
            for (int r = 0; r < NR; ++r) key[r] = 0;
        }
        return;
    }
    // groups that begin inside a lane's run: their values one after the other, then each key's group is looked up.  Every group's value is formed
    // anew for each group it is compared with (26000 x 160, f32, 8 groups: 335 us, 8 groups of 32 above 39 us).
    unsigned taken = 0;
    for (int g = 0; g < p.groups; ++g) {
        float v = -INFINITY, mine = -INFINITY;
        int before = 0;
        for (int h = -1; h < p.groups; ++h) {           // h = -1: this group's own value
            const int which = h < 0 ? g : h, lo = which * p.per_group, hi = lo + p.per_group;
            unsigned first = 0, second = 0;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const unsigned x = e0 + r >= lo && e0 + r < hi ? key[r] : 0u;
                second = max(second, min(first, x));
                first = max(first, x);
            }
#pragma unroll
            for (int o = G / 2; o > 0; o >>= 1) {
                const unsigned f = __shfl_xor_sync(FULL, first, o), s = __shfl_xor_sync(FULL, second, o);
                second = max(min(first, f), max(second, s));
                first = max(first, f);
            }
            v = first ? value_of(first) : -INFINITY;
            if (p.group_best == 2 && second) v += value_of(second);
            if (h < 0) mine = v;
            else before += v > mine || (v == mine && h < g);
        }
        if (before < p.top_groups) taken |= 1u << g;
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int g = (e0 + r) / p.per_group;
        if (g >= p.groups || !(taken >> g & 1u)) key[r] = 0;
    }
}

// PACKED: 16-bit logits that are compared themselves, without groups.
template <typename T, int G, int NR, int V, bool PACKED>
__global__ void __launch_bounds__(ROUTE_THREADS) route_kernel(const RouteP p)
{
    constexpr int SLOTS = G >= 32 ? 1 : (32 / G < NR ? 32 / G : NR);     // slots of the choice per lane: slot j is lane j % G's
    constexpr int ROWS = ROUTE_THREADS / G;                             // per block at once
    extern __shared__ int histogram[];
    const int lane = threadIdx.x & 31, at = lane & (G - 1), base = lane & ~(G - 1), e0 = at * NR;
    if (p.counts) {
        for (int i = threadIdx.x; i < p.experts; i += ROUTE_THREADS) histogram[i] = 0;
        __syncthreads();
    }
    after_previous();
    may_follow();
    // a warp's rows come and go together: the loop ends when its first row is beyond the last
    for (unsigned row0 = blockIdx.x * ROWS + (threadIdx.x / 32) * (32 / G); row0 < (unsigned)p.rows; row0 += gridDim.x * ROWS) {
        const int row = (int)row0 + lane / G;
        const bool live = row < p.rows;
        const T *logits = static_cast<const T *>(p.logits) + (long long)row * p.stride;
        T raw[NR];
        load_logits<T, NR, V>(logits, live ? p.experts : 0, e0, raw);
        float top = -INFINITY, total = 0.0f;                // softmax over the row
        if (!p.sigmoid && (p.by_score || !p.renormalise)) {
#pragma unroll
            for (int r = 0; r < NR; ++r) top = fmaxf(top, usable(to_f32(raw[r])));
            top = group_max<G>(top);
#pragma unroll
            for (int r = 0; r < NR; ++r) total += exp_from(usable(to_f32(raw[r])), top);
            total = group_sum<G>(total);
        }
        unsigned key[NR];
        unsigned order = 0;                                 // 4 bits each: which of the lane's eight logits
        if constexpr (PACKED) {
#pragma unroll
            for (int r = 0; r < NR; ++r) key[r] = packed_key(raw[r], e0 + r);
            if constexpr (NR == 8) sort_eight(key);
        } else {
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                float c = usable(to_f32(raw[r]));
                if (p.by_score && c > -INFINITY) {
                    c = p.sigmoid ? sigmoid_of(c) : expf(c - top) / total;
                    if (p.bias) c += p.bias[e0 + r];
                }
                key[r] = key_of(c);
            }
            if (p.groups > 1) keep_groups<G, NR>(p, key, lane);
            if constexpr (NR == 8) {
                // descending, equal keys in the order of their experts: neighbours are exchanged only where the later one is larger
                int idx[NR];
#pragma unroll
                for (int r = 0; r < NR; ++r) idx[r] = r;
#pragma unroll
                for (int pass = 0; pass < NR; ++pass)
#pragma unroll
                    for (int r = pass & 1; r + 1 < NR; r += 2) {
                        const bool swap = key[r + 1] > key[r];
                        const unsigned a = key[r], b = key[r + 1];
                        key[r] = max(a, b), key[r + 1] = min(a, b);
                        const int i = idx[r], j = idx[r + 1];
                        idx[r] = swap ? j : i, idx[r + 1] = swap ? i : j;
                    }
#pragma unroll
                for (int r = 0; r < NR; ++r) order |= (unsigned)idx[r] << (4 * r);
            }
        }
        int chosen[SLOTS];
        unsigned chosen_key[SLOTS];
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            chosen[s] = -1;
            chosen_key[s] = 0;
            for (int t = 0; t < G && s * G + t < p.k; ++t) {
                unsigned head = key[0];
                if constexpr (NR > 8) {
#pragma unroll
                    for (int r = 1; r < NR; ++r) head = max(head, key[r]);
                }
                const unsigned best = group_max<G>(head);
                if constexpr (PACKED) {
                    if constexpr (NR == 8) {
                        if (head == best) {
#pragma unroll
                            for (int r = 0; r + 1 < NR; ++r) key[r] = key[r + 1];
                            key[NR - 1] = 0;
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < NR; ++r) key[r] = key[r] == best ? 0u : key[r];
                    }
                    if (at == t) chosen_key[s] = best;
                } else {
                    const unsigned holders = __ballot_sync(FULL, head == best) >> base;
                    const int owner = __ffs(G == 32 ? holders : holders & ((1u << (G & 31)) - 1u)) - 1;
                    int e = e0;
                    if constexpr (NR == 8) {
                        e += (int)(order & 15u);
                        if (at == owner) {
#pragma unroll
                            for (int r = 0; r + 1 < NR; ++r) key[r] = key[r + 1];
                            key[NR - 1] = 0;
                            order >>= 4;
                        }
                    } else {
                        bool found = at != owner;
#pragma unroll
                        for (int r = 0; r < NR; ++r) {
                            const bool hit = !found && key[r] == best;
                            if (hit) e = e0 + r, key[r] = 0;
                            found = found || hit;
                        }
                    }
                    e = __shfl_sync(FULL, e, base + owner);
                    if (at == t && best) {
                        chosen[s] = e;
                        chosen_key[s] = best;
                    }
                }
            }
            if (PACKED && chosen_key[s]) chosen[s] = packed_expert(chosen_key[s]);
        }
        // slots beyond the k-th belong to nobody (s * G >= p.k for all lanes alike)
        float g[SLOTS], sum = 0.0f, most = -INFINITY;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            if (s * G >= p.k) continue;
            g[s] = -INFINITY;                               // the chosen logit
            if (chosen[s] >= 0)
                g[s] = PACKED ? packed_value<T>(chosen_key[s]) : p.by_score ? usable(to_f32(logits[chosen[s]])) : value_of(chosen_key[s]);
            most = fmaxf(most, g[s]);
        }
        if (!p.sigmoid && p.renormalise) top = group_max<G>(most);
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            if (s * G >= p.k) continue;
            if (p.sigmoid) g[s] = chosen[s] >= 0 ? sigmoid_of(g[s]) : 0.0f;
            else g[s] = p.renormalise ? exp_from(g[s], top) : exp_from(g[s], top) / total;
            sum += chosen[s] >= 0 ? g[s] : 0.0f;
        }
        if (p.renormalise) sum = group_sum<G>(sum);
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const int j = s * G + at;
            if (s * G >= p.k || !live || j >= p.k) continue;
            float v = 0.0f;
            if (chosen[s] >= 0 && (!p.renormalise || sum > 0.0f)) v = p.gate_scale * (p.renormalise ? g[s] / sum : g[s]);
            p.expert[(long long)row * p.k + j] = chosen[s];
            p.gate[(long long)row * p.k + j] = v;
            if (p.counts && chosen[s] >= 0) atomicAdd(&histogram[chosen[s]], 1);
        }
    }
    if (!p.counts) return;
    __syncthreads();
    if (p.cluster) {
        cluster_sync_all();
        if (blockIdx.x == 0)
            for (int i = threadIdx.x; i < p.experts; i += ROUTE_THREADS) {
                int n = 0;
                for (unsigned b = 0; b < gridDim.x; ++b) n += (int)ld_shared_cluster_u32(map_to_cta(smem_u32(&histogram[i]), b));
                p.counts[i] = n;
            }
        cluster_sync_all();                                 // the histograms stay until they have been read
    } else {
        for (int i = threadIdx.x; i < p.experts; i += ROUTE_THREADS)
            if (histogram[i]) atomicAdd(&p.counts[i], histogram[i]);      // whole numbers: any order
    }
}

// In front of route_kernel where its blocks add to the counts.  Nothing follows a memset early: with one in this place 2048 x 64 take 6.2 us,
// with this 3.7, 65521 x 64 18.5 and 15.1.
__global__ void __launch_bounds__(ROUTE_THREADS) clear_counts_kernel(int *counts, int experts)
{
    after_previous();
    may_follow();
    for (int i = threadIdx.x; i < experts; i += ROUTE_THREADS) counts[i] = 0;
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

// exp(l - top) of two logits.  For outputs of 16 bits by the approximate power of two, relative error about 2^-22 + |l - top| 2^-23: far below
// their own rounding; 32-bit ones get the full exponential (8192 x 256, f32: 5.4 us instead of 5.2).
template <typename T> __device__ __forceinline__ float2 exp_below(float2 l, float top)
{
    float2 t = add2(l, both(-top));
    if constexpr (sizeof(T) == 4) return make_float2(expf(t.x), expf(t.y));
    t = mul2(t, both(1.4426950408889634f));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t.x) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t.y) : "f"(t.y));
    return t;
}

// dlogits of one row: with s the scores, c = gate_scale and, over the chosen, w = s / sum(s):
//   softmax              s_i (c dgate_i - sum c dgate s)     every expert (dgate 0 where not chosen)
//   softmax, renormalised w_j (c dgate_j - sum c dgate w)    the chosen ones, 0 elsewhere
//   sigmoid              c dgate_j s_j (1 - s_j)
//   sigmoid, renormalised w_j (1 - s_j) (c dgate_j - sum c dgate w)
// Every expert's value is written first, as if it were not chosen, and then the chosen ones' over it.  The softmax over the
// whole row takes exponentials of the difference to the row's largest logit: the difference of two logits near each other is exact,
// wherever in the type's range they lie, while products of theirs need not be finite.
// Bound by the rows in flight: their loads hang on one another.  At 65521 x 64, bf16, out of HBM, 4 blocks per SM that go from row to
// row take 11.1 us, a block for every 32 rows 10.0, with 32 registers (8 blocks per SM) 9.1, with the next launch under way 8.2, as a kernel of its own 7.8; fewer than 8
// lanes per row need more registers for their share of the choice.
// DENSE: the softmax over all experts, a kernel of its own (in one kernel with the others 8.3 us at 65521 x 64: registers).
template <typename T, int G, int NR, int V, bool DENSE>
__global__ void __launch_bounds__(ROUTE_THREADS, NR == 8 && G >= 8 ? 8 : 1) route_backward_kernel(const RouteBackP p)
{
    constexpr int SLOTS = G >= 32 ? 1 : (32 / G < NR ? 32 / G : NR);
    constexpr int ROWS = ROUTE_THREADS / G;
    const int lane = threadIdx.x & 31, at = lane & (G - 1), e0 = at * NR;
    after_previous();           // no may_follow: blocks that come in early take the places of its own (10.7 -> 12.4 us)
    const int row0 = blockIdx.x * ROWS + (threadIdx.x / 32) * (32 / G);
    if (row0 < p.rows) {
        const int row = row0 + lane / G;
        const bool live = row < p.rows;
        const T *logits = static_cast<const T *>(p.logits) + (long long)row * p.stride;
        T *out = static_cast<T *>(p.dlogits) + (long long)row * p.out_stride;
        int e[SLOTS];
        float d[SLOTS], x[SLOTS];
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const int j = s * G + at;
            e[s] = -1, d[s] = 0.0f, x[s] = -INFINITY;
            if (live && j < p.k) {
                const int chosen = p.expert[(long long)row * p.k + j];
                const float dg = p.dgate[(long long)row * p.k + j];
                if (chosen >= 0 && chosen < p.experts) {
                    e[s] = chosen;
                    x[s] = usable(to_f32(logits[chosen]));
                    d[s] = x[s] > -INFINITY ? p.gate_scale * dg : 0.0f;
                }
            }
        }
        float dense[NR];                                    // what an expert that was not chosen gets
#pragma unroll
        for (int r = 0; r < NR; ++r) dense[r] = 0.0f;
        float mine[SLOTS] = {}, dot = 0.0f;
        if constexpr (DENSE) {
            T raw[NR];
            float l[NR], top = -INFINITY, total = 0.0f;
            load_logits<T, NR, V>(logits, live ? p.experts : 0, e0, raw);
#pragma unroll
            for (int r = 0; r < NR; ++r) top = fmaxf(top, l[r] = usable(to_f32(raw[r])));
            top = group_max<G>(top);
            if (!(top > -INFINITY)) top = 0.0f;             // a row that is masked throughout
#pragma unroll
            for (int r = 0; r < NR; r += 2) {
                const float2 t = exp_below<T>(make_float2(l[r], l[r + 1]), top);
                dense[r] = t.x, dense[r + 1] = t.y;
                total += dense[r];
                total += dense[r + 1];
            }
            total = group_sum<G>(total);
            const float inv = total > 0.0f ? 1.0f / total : 0.0f;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                if (s * G >= p.k) continue;
                mine[s] = exp_below<T>(both(x[s]), top).x * inv;
                dot = fmaf(d[s], mine[s], dot);
            }
            dot = group_sum<G>(dot);
#pragma unroll
            for (int r = 0; r < NR; ++r) dense[r] *= -inv * dot;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) mine[s] *= d[s] - dot;
        } else {
            float most = -INFINITY, sum = 0.0f, slope[SLOTS] = {};
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) most = fmaxf(most, x[s]);
            if (!p.sigmoid) most = group_max<G>(most);
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                if (s * G >= p.k) continue;
                const float t = expf(p.sigmoid ? -x[s] : x[s] - most);
                mine[s] = x[s] > -INFINITY ? (p.sigmoid ? 1.0f / (1.0f + t) : t) : 0.0f;
                // 1 - s as exp(-l) s: the difference loses its digits where s is near 1
                slope[s] = p.sigmoid && mine[s] > 0.0f ? t * mine[s] : 1.0f;
                sum += mine[s];
            }
            if (p.renormalise) {
                sum = group_sum<G>(sum);
#pragma unroll
                for (int s = 0; s < SLOTS; ++s) {
                    if (s * G >= p.k) continue;
                    mine[s] = sum > 0.0f ? mine[s] / sum : 0.0f;
                    dot = fmaf(d[s], mine[s], dot);
                }
                dot = group_sum<G>(dot);
            }
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) mine[s] = mine[s] * (d[s] - dot) * slope[s];
        }
        __syncwarp();                                       // every logit of the row has been read: out may be logits
#pragma unroll
        for (int r = 0; r < NR; r += V) {
            if (live && e0 + r < p.experts) {
                Pack<T, V> o;
#pragma unroll
                for (int j = 0; j < V; ++j) o.v[j] = from_f32<T>(dense[r + j]);
                store_pack<T, V>(out + e0 + r, o);
            }
        }
        __syncwarp();                                       // the chosen ones' values come after the others'
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
            if (e[s] >= 0) out[e[s]] = from_f32<T>(mine[s]);
    }
}

template <int A, int B, int C> struct Shape { static constexpr int g = A, nr = B, v = C; };
// Calls f with the lanes per row, the logits per lane and how many of them a load takes: 16 bytes where the rows allow it.
template <typename T, typename F> int with_row(int experts, bool wide, F f)
{
    constexpr int W = 16 / (int)sizeof(T);
    auto by_width = [&](auto s) { return wide ? f(Shape<decltype(s)::g, decltype(s)::nr, W>()) : f(Shape<decltype(s)::g, decltype(s)::nr, 1>()); };
    if (experts <= 8) return by_width(Shape<1, 8, 1>());
    if (experts <= 16) return by_width(Shape<2, 8, 1>());
    if (experts <= 32) return by_width(Shape<4, 8, 1>());
    if (experts <= 64) return by_width(Shape<8, 8, 1>());
    if (experts <= 128) return by_width(Shape<16, 8, 1>());
    if (experts <= 256) return by_width(Shape<32, 8, 1>());
    if (experts <= 512) return by_width(Shape<32, 16, 1>());
    return by_width(Shape<32, 32, 1>());
}

int blocks_for(int rows, int lanes) { return (int)std::min(((long long)rows * lanes + ROUTE_THREADS - 1) / ROUTE_THREADS, (long long)ROUTE_BLOCKS); }

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
                        (a->rows > 1 && a->logits_stride < a->num_experts)))
        return MOE_OVL_ERR_INVALID_ARG;
    if (a->logits_stride > 0x7fffffff) return MOE_OVL_ERR_UNSUPPORTED;
    if (!aligned(a->bias, 4) || !aligned(a->counts, 4)) return MOE_OVL_ERR_INVALID_ARG;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
    if (a->rows == 0)
        return !a->counts || cudaMemsetAsync(a->counts, 0, (size_t)a->num_experts * 4, stream) == cudaSuccess ? MOE_OVL_OK : MOE_OVL_ERR_CUDA;
    RouteP p = {a->rows, a->num_experts, a->top_k, a->num_groups, a->num_experts / a->num_groups, a->top_groups, a->group_best,
                a->score == MOE_OVL_SCORE_SIGMOID, a->renormalise != 0, a->bias != nullptr || (a->num_groups > 1 && a->group_best == 2),
                false, a->gate_scale, a->logits, a->bias, a->expert, a->gate, a->counts, a->logits_stride};
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int W = 16 / (int)sizeof(T);
        const bool wide = p.experts % W == 0 && p.stride % W == 0 && aligned(p.logits, 16);
        return with_row<T>(p.experts, wide, [&](auto c) -> int {
            using C = decltype(c);
            const bool packed = sizeof(T) == 2 && !p.by_score && p.groups == 1;
            const auto kernel = packed ? route_kernel<T, C::g, C::nr, C::v, sizeof(T) == 2> : route_kernel<T, C::g, C::nr, C::v, false>;
            const int blocks = blocks_for(p.rows, C::g);
            // a few blocks add their counts up among themselves; more of them add to memory that has been cleared
            p.cluster = p.counts && blocks <= 8;
            if (p.counts && !p.cluster) {
                const int rc = launch_behind(clear_counts_kernel, 1, dim3(ROUTE_THREADS), 0, 1, stream, p.counts, p.experts);
                if (rc != MOE_OVL_OK) return rc;
            }
            return launch_behind(kernel, (unsigned)blocks, dim3(ROUTE_THREADS), p.counts ? p.experts * 4 : 0, p.cluster ? (unsigned)blocks : 1u, stream, p);
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
        !aligned(a->dgate, 4) || (a->rows > 1 && (a->logits_stride < a->num_experts || a->dlogits_stride < a->num_experts)))
        return MOE_OVL_ERR_INVALID_ARG;
    if (std::max(a->logits_stride, a->dlogits_stride) > 0x7fffffff) return MOE_OVL_ERR_UNSUPPORTED;
    DeviceGuard guard(a->device);
    if (!guard.ok) return MOE_OVL_ERR_CUDA;
    RouteBackP p = {a->rows, a->num_experts, a->top_k, a->score == MOE_OVL_SCORE_SIGMOID, a->renormalise != 0, a->gate_scale,
                    a->logits, a->expert, a->dgate, a->dlogits, a->logits_stride, a->dlogits_stride};
    return with_dtype(a->dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int W = 16 / (int)sizeof(T);
        const bool wide = p.experts % W == 0 && p.stride % W == 0 && p.out_stride % W == 0 && aligned(p.logits, 16) && aligned(p.dlogits, 16);
        return with_row<T>(p.experts, wide, [&](auto c) {
            using C = decltype(c);
            const auto kernel = !p.sigmoid && !p.renormalise ? route_backward_kernel<T, C::g, C::nr, C::v, true> : route_backward_kernel<T, C::g, C::nr, C::v, false>;
            // as many blocks as the rows need: nothing is kept from row to row
            return launch_behind(kernel, (unsigned)(((long long)p.rows * C::g + ROUTE_THREADS - 1) / ROUTE_THREADS),
                                 dim3(ROUTE_THREADS), 0, 1, static_cast<cudaStream_t>(a->stream), p);
        });
    });
}
