// Choice of experts and the plan of their rows.
//
// route_choose_kernel: a warp takes one token at a time, lane i holding the logits of experts i, i + 32, ...  A choice is compared by a key, an
//   unsigned number of the same order (0: not to be chosen): of the logit itself where no bias and no sum of scores is involved (softmax and
//   sigmoid keep the order, so nothing is rounded), else of score + bias in double.  A pick is two or four warp
//   reductions: the largest key, then the lowest expert that has it.
//   A block takes kTokens tokens and notes who chose what in a bit per (expert, token), so that a pair's place among its expert's
//   rows is a count of bits whatever order the warps finish in, and so are the block's counts.
// route_plan_kernel: adds what lies before: the rows of lower experts, and of the expert's earlier blocks.  One block does both.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"
#include "rtn_tcgen05.cuh"

#include <float.h>

namespace rtn {

namespace {

constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr int kTokens = 128;                // of a block
constexpr int kWords = kTokens / 32;

// Numbers as unsigned of the same order, above 0.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);               // (-0 is 0)
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(double x)
{
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double value_of(uint64_t k) { return __longlong_as_double((long long)(k >> 63 ? k & 0x7fffffffffffffffull : ~k)); }

__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(0xffffffffu, k); }
__device__ __forceinline__ uint64_t warp_max(uint64_t k)
{
    const uint32_t hi = (uint32_t)(k >> 32), top = __reduce_max_sync(0xffffffffu, hi);
    return (uint64_t)top << 32 | __reduce_max_sync(0xffffffffu, hi == top ? (uint32_t)k : 0u);
}

// The largest of the warp's keys that `mine` lets take part, and the lowest index that has it (index i * 32 + lane).
template <int VPL, typename Key, typename Mine>
__device__ __forceinline__ Key best_of(const Key (&key)[VPL], int lane, int& at, Mine&& mine)
{
    Key top = 0;
    #pragma unroll
    for (int i = 0; i < VPL; ++i) if (mine(i) && key[i] > top) top = key[i];
    top = warp_max(top);
    int low = 0x7fffffff;
    #pragma unroll
    for (int i = VPL - 1; i >= 0; --i) if (mine(i) && key[i] == top) low = i * 32 + lane;
    at = (int)__reduce_min_sync(0xffffffffu, (unsigned)low);
    return top;
}

__device__ __forceinline__ double warp_sum(double x)
{
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}
__device__ __forceinline__ float warp_sum(float x)
{
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}

// Exclusive sums of n <= kMaxExperts counts in shared memory, by one warp; the total goes to sum[n].
__device__ __forceinline__ void scan_counts(const int* count, int* sum, int n, int lane)
{
    int before = 0;
    for (int e0 = 0; e0 < n; e0 += 32) {
        const int c = e0 + lane < n ? count[e0 + lane] : 0;
        int x = c;
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (e0 + lane < n) sum[e0 + lane] = before + x - c;
        before += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) sum[n] = before;
}

// counts: [blocks][E], or NULL: no plan, or one block, which finishes it.
template <typename T, int VPL, bool kWide>
__global__ void __launch_bounds__(kThreads)
route_choose_kernel(const RouteArgs g, int* counts)
{
    using Key = typename std::conditional<kWide, uint64_t, uint32_t>::type;
    extern __shared__ uint32_t chosen[];                       // [E][kWords]; then count and start, [E + 1] each
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t t0 = (int64_t)blockIdx.x * kTokens;
    const int n_tok = g.T - t0 < kTokens ? (int)(g.T - t0) : kTokens;
    const bool plan = g.start != nullptr;
    const int k = g.top_k;
    if (plan) {
        for (int i = threadIdx.x; i < g.E * kWords; i += kThreads) chosen[i] = 0;
        __syncthreads();
    }
    const int per_group = g.E / g.groups;
    for (int t = warp; t < n_tok; t += kWarps) {
        const T* row = static_cast<const T*>(g.logits) + (t0 + t) * g.stride;
        float x[VPL];
        Key key[VPL];
        #pragma unroll
        for (int i = 0; i < VPL; ++i) x[i] = i * 32 + lane < g.E ? to_f32(row[i * 32 + lane]) : -INFINITY;
        float top = -INFINITY;
        #pragma unroll
        for (int i = 0; i < VPL; ++i) {
            if (!(x[i] > -INFINITY)) x[i] = -INFINITY;         // NaN
            x[i] = fminf(x[i], FLT_MAX);
            top = fmaxf(top, x[i]);
        }
        {
            const uint32_t u = warp_max(key_of(top));
            top = __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u);
        }
        float sum = 1.f;                                        // of a softmax over all experts
        if constexpr (kWide) {
            double s[VPL], all = 0.0;
            #pragma unroll
            for (int i = 0; i < VPL; ++i) {
                s[i] = g.score == RTN_SCORE_SIGMOID ? 1.0 / (1.0 + exp(-(double)x[i])) : x[i] == -INFINITY ? 0.0 : exp((double)x[i] - (double)top);
                all += s[i];
            }
            all = g.score == RTN_SCORE_SIGMOID ? 1.0 : warp_sum(all);
            sum = (float)all;
            #pragma unroll
            for (int i = 0; i < VPL; ++i) {
                const float b = g.bias != nullptr && i * 32 + lane < g.E ? g.bias[i * 32 + lane] : 0.f;
                key[i] = x[i] > -INFINITY && b > -INFINITY ? key_of(s[i] / all + (double)b) : 0;
            }
        } else {
            #pragma unroll
            for (int i = 0; i < VPL; ++i) key[i] = x[i] > -INFINITY ? key_of(x[i]) : 0;
            if (g.score == RTN_SCORE_SOFTMAX && !g.renormalise) {
                float all = 0.f;
                #pragma unroll
                for (int i = 0; i < VPL; ++i) all += x[i] > -INFINITY ? expf(x[i] - top) : 0.f;
                sum = warp_sum(all);
            }
        }
        if (g.groups > 1) {
            Key mine[1] = {0};                                  // lane i: the value of group i
            for (int gr = 0; gr < g.groups; ++gr) {
                const int lo = gr * per_group, hi = lo + per_group;
                int at = 0;
                Key best = best_of(key, lane, at, [&](int i) { return i * 32 + lane >= lo && i * 32 + lane < hi; });
                if constexpr (kWide) {
                    if (g.group_top > 1 && best != 0) {
                        double value = value_of(best);
                        uint64_t limit = best;
                        int last = at;                          // the picks go down by (key, index)
                        for (int n = 1; n < g.group_top; ++n) {
                            const uint64_t next = best_of(key, lane, at, [&](int i) {
                                const int e = i * 32 + lane;
                                return e >= lo && e < hi && (key[i] < limit || (key[i] == limit && e > last));
                            });
                            if (next == 0) break;
                            value += value_of(next);
                            limit = next; last = at;
                        }
                        best = key_of(value);
                    }
                }
                if (lane == gr) mine[0] = best;
            }
            uint32_t kept = 0;
            for (int n = 0; n < g.kept; ++n) {
                int at = 0;
                if (best_of(mine, lane, at, [&](int) { return true; }) == 0) break;
                kept |= 1u << at;
                if (lane == at) mine[0] = 0;
            }
            #pragma unroll
            for (int i = 0; i < VPL; ++i) {
                const int e = i * 32 + lane;
                if (e < g.E && !(kept >> (e / per_group) & 1u)) key[i] = 0;
            }
        }
        int pick = -1;                                          // lane j: choice j and its logit
        float logit = -INFINITY;
        for (int j = 0; j < k; ++j) {
            int at = 0;
            if (best_of(key, lane, at, [&](int) { return true; }) == 0) break;
            float v = 0.f;
            #pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (i * 32 + lane == at) { v = x[i]; key[i] = 0; }
            v = __shfl_sync(0xffffffffu, v, at & 31);
            if (lane == j) { pick = at; logit = v; }
        }
        float w = 0.f;
        if (g.renormalise) {
            // s up to a factor that all choices share, so that scores too small for fp32 still have their ratios
            const uint32_t u = warp_max(key_of(logit));
            const float best = __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u);
            if (pick >= 0)
                w = g.score == RTN_SCORE_SOFTMAX ? expf(logit - best) : expf(fminf(logit, 0.f) - fminf(best, 0.f)) / (1.f + expf(-fabsf(logit)));
            const float all = warp_sum(w);
            if (pick >= 0) w /= all;
        } else if (pick >= 0) {
            w = g.score == RTN_SCORE_SOFTMAX ? expf(logit - top) / sum : 1.f / (1.f + expf(-logit));
        }
        if (lane < k) {
            g.experts[(t0 + t) * k + lane] = pick;
            g.weights[(t0 + t) * k + lane] = w * g.scale;
            if (plan && pick >= 0) atomicOr(&chosen[pick * kWords + (t >> 5)], 1u << (t & 31));
        }
    }
    if (!plan) return;
    int* count = reinterpret_cast<int*>(chosen + g.E * kWords);
    int* start = count + g.E + 1;
    __syncthreads();
    const bool alone = counts == nullptr;
    for (int e = threadIdx.x; e < g.E; e += kThreads) {
        int n = 0;
        #pragma unroll
        for (int i = 0; i < kWords; ++i) n += __popc(chosen[e * kWords + i]);
        count[e] = n;
        if (!alone) counts[(int64_t)blockIdx.x * g.E + e] = n;
    }
    if (alone) {
        __syncthreads();
        if (warp == 0) scan_counts(count, start, g.E, lane);
        __syncthreads();
        for (int e = threadIdx.x; e <= g.E; e += kThreads) g.start[e] = start[e];
    }
    for (int i = threadIdx.x; i < n_tok * k; i += kThreads) {
        const int t = i / k, e = g.experts[t0 * k + i];
        int at = -1;
        if (e >= 0) {
            at = 0;
            for (int j = 0; j < (t >> 5); ++j) at += __popc(chosen[e * kWords + j]);
            at += __popc(chosen[e * kWords + (t >> 5)] & ((1u << (t & 31)) - 1u));
            if (alone) { at += start[e]; g.tokens[at] = (int)(t0 + t); }
        }
        g.place[t0 * k + i] = at;
    }
    tc::pdl_trigger();
}

__global__ void __launch_bounds__(kThreads)
route_plan_kernel(const RouteArgs g, const int* counts, int blocks)
{
    extern __shared__ int sums[];                               // total, before, start: [E + 1] each
    int *total = sums, *before = sums + g.E + 1, *start = before + g.E + 1;
    for (int e = threadIdx.x; e < g.E; e += kThreads) total[e] = before[e] = 0;
    tc::pdl_wait();
    __syncthreads();
    const int parts = g.E < kThreads ? kThreads / g.E : 1;
    for (int i = threadIdx.x; i < g.E * parts; i += kThreads) {
        const int e = i % g.E, p = i / g.E;
        int a = 0, b = 0;
        #pragma unroll 8
        for (int j = p; j < blocks; j += parts) {
            const int c = counts[(int64_t)j * g.E + e];
            a += c;
            b += j < (int)blockIdx.x ? c : 0;
        }
        atomicAdd(&total[e], a);
        atomicAdd(&before[e], b);
    }
    __syncthreads();
    if (threadIdx.x < 32) scan_counts(total, start, g.E, threadIdx.x);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= g.E; e += kThreads) g.start[e] = start[e];
    const int64_t t0 = (int64_t)blockIdx.x * kTokens;
    const int k = g.top_k, n = (int)((g.T - t0 < kTokens ? g.T - t0 : kTokens) * k);
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int e = g.experts[t0 * k + i];
        if (e < 0) continue;
        const int at = g.place[t0 * k + i] + start[e] + before[e];
        g.place[t0 * k + i] = at;
        g.tokens[at] = (int)(t0 + i / k);
    }
}

template <typename T, int VPL>
cudaError_t launch_choose(const RouteArgs& g, int* counts, unsigned blocks, cudaStream_t s)
{
    const size_t smem = g.start != nullptr ? (size_t)g.E * kWords * 4 + 2 * (g.E + 1) * 4 : 0;
    // scores have to be computed where a bias or a sum of them is compared
    if (g.bias != nullptr || (g.groups > 1 && g.group_top > 1)) route_choose_kernel<T, VPL, true><<<blocks, kThreads, smem, s>>>(g, counts);
    else route_choose_kernel<T, VPL, false><<<blocks, kThreads, smem, s>>>(g, counts);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_route_experts(const RouteArgs& g, cudaStream_t s)
{
    if (g.T == 0) return cudaMemsetAsync(g.start, 0, (size_t)(g.E + 1) * sizeof(int32_t), s);
    const int64_t blocks = (g.T + kTokens - 1) / kTokens;
    void* counts = nullptr;
    if (g.start != nullptr && blocks > 1) {
        const cudaError_t e = scratch_alloc(&counts, (size_t)blocks * g.E * sizeof(int), s);
        if (e != cudaSuccess) return e;
    }
    int* c = static_cast<int*>(counts);
    cudaError_t e = with_dtype(g.dtype, [&](auto t) {
        using T = decltype(t);
        if (g.E <= 32) return launch_choose<T, 1>(g, c, (unsigned)blocks, s);
        if (g.E <= 64) return launch_choose<T, 2>(g, c, (unsigned)blocks, s);
        if (g.E <= 128) return launch_choose<T, 4>(g, c, (unsigned)blocks, s);
        if (g.E <= 256) return launch_choose<T, 8>(g, c, (unsigned)blocks, s);
        if (g.E <= 512) return launch_choose<T, 16>(g, c, (unsigned)blocks, s);
        return launch_choose<T, 32>(g, c, (unsigned)blocks, s);
    });
    if (e == cudaSuccess && counts != nullptr)
        e = launch_pdl(route_plan_kernel, dim3((unsigned)blocks), dim3(kThreads), (size_t)3 * (g.E + 1) * sizeof(int), s, g, (const int*)counts, (int)blocks);
    if (counts != nullptr) {
        const cudaError_t e2 = cudaFreeAsync(counts, s);
        if (e == cudaSuccess) e = e2;
    }
    return e;
}

}  // namespace rtn
