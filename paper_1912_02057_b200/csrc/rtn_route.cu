// Choice of experts and the plan of their rows.
//
// route_choose_kernel: a warp takes one token at a time, a lane VPL experts side by side.  A choice is compared by a key, an unsigned number
//   of the same order (0: not to be chosen): of the logit itself where no bias and no sum of scores is involved (softmax and sigmoid keep the
//   order, so nothing is rounded), else of score + bias in fp32.  There two neighbours in the order that are nearer to each other than their
//   rounding errors make the warp choose this token's experts again in double (of ordinary tokens a few in a thousand), and what double leaves
//   open, scores next to 1 or under large biases, in pairs of doubles when the block's other tokens are done (16384 tokens, 8 of 128, bias: 30.7
//   us without that, 32.7 with it).
//   A pick is one warp reduction and one vote: the largest key, and the first lane that has it.  Groups are looked at all at once, a group's
//   lanes side by side, where their sizes let them be, else one after the other.
//   A block notes who chose what in a bit per (expert, token), so that a pair's place among its expert's rows is a count of bits
//   whatever order the warps finish in, and so are the block's counts.
// route_plan_kernel adds what lies before: the rows of lower experts, and of the expert's earlier blocks.  One block does both.
// route_list_kernel does the first kernel's work for many tokens.
// Bound: latency (a launch and dependent loads) for a token.  For a batch the instructions of a token and where they run: 96 tokens, 8 of 256 in 4 of 8 groups, with a
// bias take 1660 warp instructions each, on six blocks of 16 warps, so that four warps share a scheduler of six SMs (0.44 of its issue slots) and the other SMs
// have nothing to do.  For many tokens the places of the lists, each of which every logit goes through, and a round of blocks that comes out uneven (256 on 148
// SMs; 0.44 of the issue slots).
// Measured (one B200, in a graph): one token, 4 of 64 experts 3.4 us; 96 tokens as above 10.9 us; 16384 tokens, 8 of 128 12.6 us (4.2 MB of logits: 0.6 us at
// the copy rate).  What leaves the lists: a bias or sums of scores, whose fp32 values need the bound and the exact form, groups, and more than
// eight choices, the places that a list has; 16384 tokens take, a warp to each, 8 of 128 with a bias 32.7 us, 12 of 128 28.2, 8 of 256 with a bias 51.6, in 4 of 8
// groups by sums of two 64.1, of three (all in double) 251.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"
#include "rtn_tcgen05.cuh"

#include <float.h>
#include <type_traits>

namespace rtn {

namespace {

constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxTokens = 128;             // of a block
constexpr int kList = 8, kShare = 4;        // a thread's list of a token's best; threads that share a token
constexpr int kListTokens = 64, kListThreads = kListTokens * kShare;       // of a block
constexpr int64_t kListFrom = 4096;         // tokens
constexpr int kScanBlocks = 32;             // more: the counts are added up ahead (each block by itself reads them all)
constexpr float kUnit = 5.9604644775390625e-8f;                // 2^-24

// Numbers as unsigned of the same order, above 0.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);               // (-0 is 0)
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
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
__device__ __forceinline__ float warp_max(float x) { return value_of(warp_max(key_of(x))); }

template <typename F>
__device__ __forceinline__ F warp_sum(F x)
{
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}

// The logits of a lane's experts as they are in memory, asked for ahead.
template <typename T, int VPL>
__device__ __forceinline__ void ask_logits(const RouteArgs& g, int64_t t, int lane, T (&raw)[VPL])
{
    const T* row = static_cast<const T*>(g.logits) + t * g.stride + lane * VPL;
    constexpr int kBytes = VPL * (int)sizeof(T), kVec = kBytes % 16 == 0 ? 16 : kBytes % 8 == 0 ? 8 : kBytes % 4 == 0 ? 4 : 2;
    if (kVec > (int)sizeof(T) && g.E % VPL == 0 && (reinterpret_cast<uintptr_t>(row) & (kVec - 1)) == 0) {
        if (lane * VPL < g.E) {
            #pragma unroll
            for (int i = 0; i < kBytes / kVec; ++i) {
                if constexpr (kVec == 16) reinterpret_cast<uint4*>(raw)[i] = reinterpret_cast<const uint4*>(row)[i];
                else if constexpr (kVec == 8) reinterpret_cast<uint2*>(raw)[i] = reinterpret_cast<const uint2*>(row)[i];
                else if constexpr (kVec == 4) reinterpret_cast<uint32_t*>(raw)[i] = reinterpret_cast<const uint32_t*>(row)[i];
            }
        }
    } else {
        #pragma unroll
        for (int i = 0; i < VPL; ++i) raw[i] = row[lane * VPL + i < g.E ? i : -lane * VPL];           // (behind the last: the first)
    }
}
// NaN as -inf, +inf as the largest number.
template <typename T, int VPL>
__device__ __forceinline__ void take_logits(const RouteArgs& g, int lane, const T (&raw)[VPL], float (&x)[VPL])
{
    #pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const float v = to_f32(raw[i]);
        x[i] = lane * VPL + i < g.E && v > -INFINITY ? fminf(v, FLT_MAX) : -INFINITY;
    }
}

// Lane j: choice j and its logit.
struct Choice { int pick; float logit; };
constexpr int kOpen = -2;                   // (of all lanes) not decided

// The largest of the warp's keys that `mine` lets take part, and the lowest index that has it.
template <int VPL, typename Mine>
__device__ __forceinline__ uint64_t best_of(const uint64_t (&key)[VPL], int lane, int& at, Mine&& mine)
{
    uint64_t top = 0;
    #pragma unroll
    for (int i = 0; i < VPL; ++i) if (mine(i) && key[i] > top) top = key[i];
    top = warp_max(top);
    int low = 0x7fffffff;
    #pragma unroll
    for (int i = VPL - 1; i >= 0; --i) if (mine(i) && key[i] == top) low = lane * VPL + i;
    at = (int)__reduce_min_sync(0xffffffffu, (unsigned)low);
    return top;
}

// Weights of a token's choices (top and sum: of a softmax over all experts, where it is not renormalised), and the note of who chose what.
__device__ __forceinline__ void finish_token(const RouteArgs& g, int64_t t, const Choice& c, float top, float sum, uint32_t* chosen, int words, int bit)
{
    const int lane = threadIdx.x & 31;
    float w = 0.f;
    if (g.renormalise) {
        // s up to a factor that all choices share, so that scores too small for fp32 still have their ratios
        const float best = warp_max(c.logit);
        if (c.pick >= 0)
            w = g.score == RTN_SCORE_SOFTMAX ? expf(c.logit - best) : expf(fminf(c.logit, 0.f) - fminf(best, 0.f)) / (1.f + expf(-fabsf(c.logit)));
        const float all = warp_sum(w);
        if (c.pick >= 0) w /= all;
    } else if (c.pick >= 0) {
        w = g.score == RTN_SCORE_SOFTMAX ? expf(c.logit - top) / sum : 1.f / (1.f + expf(-c.logit));
    }
    if (lane < g.top_k) {
        g.experts[t * g.top_k + lane] = c.pick;
        g.weights[t * g.top_k + lane] = w * g.scale;
        if (chosen != nullptr && c.pick >= 0) atomicOr(&chosen[c.pick * words + (bit >> 5)], 1u << (bit & 31));
    }
}

// A sum of two doubles as a pair: the rounded sum, and what it left out (0 beside an infinity).
struct Pair { double hi, lo; };
__device__ __forceinline__ Pair pair_sum(double a, double b)
{
    const double s = a + b, t = s - a;
    return Pair{s, isinf(s) ? 0.0 : (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ Pair pair_sum(Pair a, Pair b)
{
    const Pair s = pair_sum(a.hi, b.hi);
    return pair_sum(s.hi, s.lo + (a.lo + b.lo));
}
// Places in the order of choices: by c, as a pair, by the logit, which a score grows with where c does not tell any more, and by the index, lowest first.  Of
// infinities nothing but the index counts.
struct Place { uint64_t hi, lo; uint32_t logit; int at; };
__device__ __forceinline__ bool ahead(const Place& a, const Place& b)
{
    if (a.hi != b.hi) return a.hi > b.hi;
    if (a.lo != b.lo) return a.lo > b.lo;
    return a.logit != b.logit ? a.logit > b.logit : a.at < b.at;
}
// The first of the lanes' places (at -1: there is none).
__device__ __forceinline__ Place first_of(Place p)
{
    const uint64_t hi = warp_max(p.at >= 0 ? p.hi : 0);
    bool same = p.at >= 0 && p.hi == hi;
    const uint64_t lo = warp_max(same ? p.lo : 0);
    same = same && p.lo == lo;
    const uint32_t logit = warp_max(same ? p.logit : 0u);
    same = same && p.logit == logit;
    return Place{hi, lo, logit, (int)__reduce_min_sync(0xffffffffu, same ? (unsigned)p.at : 0xffffffffu)};
}
// Expert e's place (0 for hi: not to be chosen).  top, all: the largest logit and the sum of exponentials of a softmax.  A sigmoid next to 1 is 1 less what it
// lacks, so that neither end hides a difference.
template <typename T>
__device__ __noinline__ Place place_of(const RouteArgs& g, int64_t t, int e, double top, double all)
{
    const float v = to_f32(static_cast<const T*>(g.logits)[t * g.stride + e]), x = v > -INFINITY ? fminf(v, FLT_MAX) : -INFINITY;
    const float b = g.bias != nullptr ? g.bias[e] : 0.f;
    if (!(x > -INFINITY && b > -INFINITY)) return Place{0, 0, 0, e};
    Pair c{(double)b, 0.0};
    if (g.score == RTN_SCORE_SIGMOID) {
        const double r = exp(-fabs((double)x)), s = r / (1.0 + r);
        c = x > 0.f ? pair_sum(pair_sum(c.hi, 1.0), Pair{-s, 0.0}) : pair_sum(c.hi, s);
    } else c = pair_sum(c.hi, exp((double)x - top) / all);
    return Place{key_of(c.hi), key_of(c.lo), isinf(c.hi) ? 0u : key_of(x), e};
}
// The first place behind `last` of experts lo .. hi - 1 (of the groups in `kept`).  Rolled up and worked out again each time: it is to need no more registers than the
// kernel has, and hardly a token comes here.
template <typename T>
__device__ __noinline__ Place next_place(const RouteArgs& g, int64_t t, int lo, int hi, uint32_t kept, const Place& last, double top, double all)
{
    Place best{0, 0, 0, -1};
    #pragma unroll 1
    for (int e = lo + (threadIdx.x & 31); e < hi; e += 32) {
        if (!(kept >> (e / (g.E / g.groups)) & 1u)) continue;
        const Place p = place_of<T>(g, t, e, top, all);
        if (p.hi != 0 && ahead(last, p) && (best.at < 0 || ahead(p, best))) best = p;
    }
    __syncwarp();
    return first_of(best);
}

// One token, for any groups, where double does not tell two choices apart.  (A softmax's sum is off by up to 2^-48, for all scores alike.)
template <typename T>
__device__ __noinline__ void choose_by_pairs(const RouteArgs& g, int64_t t, uint32_t* chosen, int words, int bit)
{
    const int lane = threadIdx.x & 31, per_group = g.E / g.groups;
    const T* row = static_cast<const T*>(g.logits) + t * g.stride;
    float most = -INFINITY;
    #pragma unroll 1
    for (int e = lane; e < g.E; e += 32) most = fmaxf(most, to_f32(row[e]));       // (a NaN is never the larger)
    const float top = fminf(warp_max(most), FLT_MAX);
    double all = 0.0;
    #pragma unroll 1
    for (int e = lane; e < g.E; e += 32) {
        const float x = to_f32(row[e]);
        if (x > -INFINITY) all += exp((double)fminf(x, FLT_MAX) - (double)top);
    }
    all = warp_sum(all);
    const Place before{~0ull, ~0ull, ~0u, -1};
    uint32_t kept = 0xffffffffu;
    if (g.groups > 1) {
        Place value{0, 0, 0, -1};                               // lane i: of group i
        #pragma unroll 1
        for (int gr = 0; gr < g.groups; ++gr) {
            Place last = before;
            Pair sum{0.0, 0.0};
            int n = 0;
            #pragma unroll 1
            for (; n < g.group_top; ++n) {
                last = next_place<T>(g, t, gr * per_group, (gr + 1) * per_group, kept, last, top, all);
                if (last.at < 0) break;
                const Pair c{value_of(last.hi), value_of(last.lo)};
                sum = n == 0 ? c : pair_sum(sum, c);
            }
            if (lane == gr && n > 0) value = Place{key_of(sum.hi), key_of(sum.lo), 0u, gr};
        }
        kept = 0;
        #pragma unroll 1
        for (int n = 0; n < g.kept; ++n) {
            const Place best = first_of(value);
            if (best.at < 0) break;
            kept |= 1u << best.at;
            if (lane == best.at) value.at = -1;
        }
    }
    Choice c{-1, -INFINITY};
    Place last = before;
    #pragma unroll 1
    for (int j = 0; j < g.top_k; ++j) {
        last = next_place<T>(g, t, 0, g.E, kept, last, top, all);
        if (last.at < 0) break;
        if (lane == j) { c.pick = last.at; c.logit = fminf(to_f32(row[last.at]), FLT_MAX); }
    }
    finish_token(g, t, c, top, (float)all, chosen, words, bit);
}

// One token's choices in double, for any groups.  Its own errors are below 2^-50 of score and c; two neighbours in the order that are nearer than a few of
// those, and not the same logit and bias, are left to the form above (kOpen): scores next to 1, or under a large bias.
template <typename T, int VPL>
__device__ __noinline__ Choice choose_exact(const RouteArgs& g, int64_t t)
{
    const int lane = threadIdx.x & 31;
    constexpr double kNear = 0x1p-47;
    float x[VPL];
    alignas(16) T raw[VPL];
    ask_logits<T, VPL>(g, t, lane, raw);
    take_logits<T, VPL>(g, lane, raw, x);
    float most = -INFINITY;
    #pragma unroll
    for (int i = 0; i < VPL; ++i) most = fmaxf(most, x[i]);
    const double top = warp_max(most);
    uint64_t key[VPL];
    double s[VPL], all = 0.0;
    #pragma unroll
    for (int i = 0; i < VPL; ++i) {
        s[i] = g.score == RTN_SCORE_SIGMOID ? 1.0 / (1.0 + exp(-(double)x[i])) : x[i] == -INFINITY ? 0.0 : exp((double)x[i] - top);
        all += s[i];
    }
    all = g.score == RTN_SCORE_SIGMOID ? 1.0 : warp_sum(all);
    float most_bias = 0.f;
    #pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const float b = g.bias != nullptr && lane * VPL + i < g.E ? g.bias[lane * VPL + i] : 0.f;
        key[i] = x[i] > -INFINITY && b > -INFINITY ? key_of(s[i] / all + (double)b) : 0;
        if (key[i] != 0 && b < INFINITY) most_bias = fmaxf(most_bias, fabsf(b));
    }
    const double reach = warp_max(most_bias);
    bool unsure = false;
    if (g.groups > 1) {
        const int per_group = g.E / g.groups;
        uint64_t value_key[1] = {0};                            // lane i: the value of group i
        for (int gr = 0; gr < g.groups; ++gr) {
            const int lo = gr * per_group, hi = lo + per_group;
            int at = 0;
            uint64_t best = best_of(key, lane, at, [&](int i) { return lane * VPL + i >= lo && lane * VPL + i < hi; });
            if (g.group_top > 1 && best != 0) {
                double value = value_of(best);
                uint64_t limit = best;
                int last = at;                                  // the picks go down by (key, index)
                for (int n = 1; n < g.group_top; ++n) {
                    const uint64_t next = best_of(key, lane, at, [&](int i) {
                        const int e = lane * VPL + i;
                        return e >= lo && e < hi && (key[i] < limit || (key[i] == limit && e > last));
                    });
                    if (next == 0) break;
                    value += value_of(next);
                    limit = next; last = at;
                }
                best = key_of(value);
            }
            if (lane == gr) value_key[0] = best;
        }
        uint32_t kept = 0;
        double last = INFINITY;
        for (int n = 0; n < g.kept; ++n) {
            int at = 0;
            const uint64_t best = best_of(value_key, lane, at, [&](int) { return true; });
            if (best == 0) break;
            kept |= 1u << at;
            last = value_of(best);
            if (lane == at) value_key[0] = 0;
        }
        // the last that is kept and those that are not (a sum's terms are no larger than it and twice their biases)
        const double size = 2.0 * fabs(last) + 4.0 * g.group_top * reach;
        unsure = __any_sync(0xffffffffu, value_key[0] != 0 && !(last - value_of(value_key[0]) > kNear * size));
        #pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int e = lane * VPL + i;
            if (e < g.E && !(kept >> (e / per_group) & 1u)) key[i] = 0;
        }
    }
    Choice c{-1, -INFINITY};
    uint64_t before = 0;                                        // the last choice
    float before_logit = 0.f;
    int before_at = 0;
    auto near = [&](uint64_t next, double size) {
        const double a = value_of(before), b = value_of(next);
        return !(a - b > kNear * (fabs(a) + fabs(b) + size));
    };
    auto look = [&](uint64_t next, int at, float logit) {
        if (before == 0 || !near(next, 4.0 * reach)) return;
        const float b = g.bias != nullptr ? g.bias[at] : 0.f, before_b = g.bias != nullptr ? g.bias[before_at] : 0.f;
        unsure = unsure || ((logit != before_logit || b != before_b) && near(next, 2.0 * (fabs((double)b) + fabs((double)before_b))));
    };
    auto take = [&](float& logit, int& at) {                    // the best that is left
        const uint64_t best = best_of(key, lane, at, [&](int) { return true; });
        if (best == 0) return best;
        #pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (lane * VPL + i == at) { logit = x[i]; key[i] = 0; }
        logit = __shfl_sync(0xffffffffu, logit, at / VPL);
        look(best, at, logit);
        return best;
    };
    #pragma unroll 1
    for (int j = 0; j < g.top_k; ++j) {
        int at = 0;
        float logit = 0.f;
        const uint64_t best = take(logit, at);
        if (best == 0) break;
        if (lane == j) { c.pick = at; c.logit = logit; }
        before = best; before_logit = logit; before_at = at;
    }
    uint64_t left = 0;
    #pragma unroll
    for (int i = 0; i < VPL; ++i) left = key[i] > left ? key[i] : left;
    left = warp_max(left);
    if (before != 0 && left != 0 && near(left, 4.0 * reach)) {
        int at = 0;
        float logit = 0.f;
        take(logit, at);
    }
    if (unsure) c.pick = kOpen;
    return c;
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

// The block's part of the plan, from who chose what: counts: [blocks][E], or NULL: there is one block, which finishes it.  Behind the choices and their
// notes, called by all.  chosen: [E][words]; behind it count and start, [E + 1] each.
__device__ __forceinline__ void note_block(const RouteArgs& g, uint32_t* chosen, int64_t t0, int n_tok, int words, int* counts)
{
    tc::pdl_trigger();
    const int k = g.top_k, threads = (int)blockDim.x;
    int* count = reinterpret_cast<int*>(chosen + g.E * words);
    int* start = count + g.E + 1;
    __syncthreads();
    const bool alone = counts == nullptr;
    for (int e = threadIdx.x; e < g.E; e += threads) {
        int n = 0;
        for (int i = 0; i < words; ++i) n += __popc(chosen[e * words + i]);
        count[e] = n;
        if (!alone) counts[(int64_t)blockIdx.x * g.E + e] = n;
    }
    if (alone) {
        __syncthreads();
        if (threadIdx.x < 32) scan_counts(count, start, g.E, threadIdx.x);
        __syncthreads();
        for (int e = threadIdx.x; e <= g.E; e += threads) g.start[e] = start[e];
    }
    for (int i = threadIdx.x; i < n_tok * k; i += threads) {
        const int t = i / k, e = g.experts[t0 * k + i];
        int at = -1;
        if (e >= 0) {
            at = 0;
            for (int j = 0; j < (t >> 5); ++j) at += __popc(chosen[e * words + j]);
            at += __popc(chosen[e * words + (t >> 5)] & ((1u << (t & 31)) - 1u));
            if (alone) { at += start[e]; g.tokens[at] = (int)(t0 + t); }
        }
        g.place[t0 * k + i] = at;
    }
}

// What a launch is told: tokens of a block, experts of a group; whether the groups' lanes are side by side, 2^group_shift of them (else 1).
struct RoutePlan { int tokens, group_size, group_shift; bool side_by_side; };

// counts: [blocks][E], or NULL: no plan, or one block, which finishes it.  kScored: a bias or sums of scores.  (Two blocks to an SM, and tokens
// that double leaves open only when the others are done: what is called for one in a thousand is not to take the others' registers.)
template <typename T, int VPL, bool kScored>
__global__ void __launch_bounds__(kThreads, kScored && VPL <= 4 ? 2 : 1)
route_choose_kernel(const __grid_constant__ RouteArgs g, const RoutePlan p, int* counts)
{
    extern __shared__ uint32_t chosen[];                       // [E][words]; then count and start, [E + 1] each
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, words = (p.tokens + 31) / 32;
    const int64_t t0 = (int64_t)blockIdx.x * p.tokens;
    const int n_tok = g.T - t0 < p.tokens ? (int)(g.T - t0) : p.tokens;
    const bool plan = g.start != nullptr;
    const int k = g.top_k;
    tc::pdl_wait();
    float bias[VPL];
    #pragma unroll
    for (int i = 0; i < VPL; ++i) bias[i] = kScored && g.bias != nullptr && lane * VPL + i < g.E ? g.bias[lane * VPL + i] : 0.f;
    if (plan) {
        for (int i = threadIdx.x; i < g.E * words; i += kThreads) chosen[i] = 0;
        __syncthreads();
    }
    alignas(16) T raw[VPL];
    if (warp < n_tok) ask_logits<T, VPL>(g, t0 + warp, lane, raw);
    uint32_t open = 0;                                          // this warp's tokens that double leaves open
    for (int t = warp; t < n_tok; t += kWarps) {
        float x[VPL];
        take_logits<T, VPL>(g, lane, raw, x);
        if (t + kWarps < n_tok) ask_logits<T, VPL>(g, t0 + t + kWarps, lane, raw);
        float top = -INFINITY, sum = 1.f;                       // of a softmax over all experts
        uint32_t key[VPL];
        float slack = 0.f;                                      // how far a c (of this lane's) may be off
        if (g.score == RTN_SCORE_SOFTMAX && (kScored || !g.renormalise)) {
            #pragma unroll
            for (int i = 0; i < VPL; ++i) top = fmaxf(top, x[i]);
            top = warp_max(top);
            float all = 0.f;
            #pragma unroll
            for (int i = 0; i < VPL; ++i) all += x[i] > -INFINITY ? __expf(x[i] - top) : 0.f;
            sum = warp_sum(all);
        }
        if constexpr (kScored) {
            // A score's error in units of 2^-24.  Sigmoid: (2 |x| + 4) (1 - s) s <= 1.5 for the exponential, 2 s for sum and quotient.  Softmax with
            // d = top - x: (2 d + 4) s <= 5, the sum's (VPL + 5 adds of terms with as much) and the quotient's 4.
            const float units = g.score == RTN_SCORE_SIGMOID ? 3.5f : (float)VPL + 24.f;
            const float inverse = 1.f / sum;
            #pragma unroll
            for (int i = 0; i < VPL; ++i) {
                const float s = g.score == RTN_SCORE_SIGMOID ? 1.f / (1.f + __expf(-x[i])) : __expf(x[i] - top) * inverse;
                key[i] = x[i] > -INFINITY && bias[i] > -INFINITY ? key_of(s + bias[i]) : 0;
                if (key[i] != 0) slack = fmaxf(slack, fabsf(bias[i]));
            }
            slack = kUnit * (units + 1.f) * 1.1f * (1.f + warp_max(slack));
        } else {
            #pragma unroll
            for (int i = 0; i < VPL; ++i) key[i] = x[i] > -INFINITY ? key_of(x[i]) : 0;
        }
        bool unsure = g.groups > 1 && g.group_top > 2;             // (scored)
        if (g.groups > 1 && !unsure) {
            uint32_t a = 0, b = 0;                              // the largest and second largest of this lane's group
            int mine = lane >> p.group_shift;
            if (p.side_by_side) {
                #pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    b = max(b, min(a, key[i]));
                    a = max(a, key[i]);
                }
                for (int d = 1; d < 1 << p.group_shift; d <<= 1) {
                    const uint32_t c = __shfl_xor_sync(0xffffffffu, a, d), e = __shfl_xor_sync(0xffffffffu, b, d);
                    b = max(max(b, e), min(a, c));
                    a = max(a, c);
                }
            } else {                                            // one group after the other; lane i has group i
                mine = lane;
                for (int gr = 0, lo = -lane * VPL; gr < g.groups; ++gr, lo += p.group_size) {
                    uint32_t c = 0, e = 0;
                    #pragma unroll
                    for (int i = 0; i < VPL; ++i)
                        if (i >= lo && i < lo + p.group_size) { e = max(e, min(c, key[i])); c = max(c, key[i]); }
                    const uint32_t first = warp_max(c);
                    const int from = __ffs(__ballot_sync(0xffffffffu, c == first)) - 1;
                    const uint32_t second = warp_max(lane == from ? e : c);
                    if (lane == gr) { a = first; b = second; }
                }
            }
            if (g.group_top == 2 && b != 0) a = key_of(value_of(a) + value_of(b));
            if (mine >= g.groups) a = 0;
            uint32_t last = 0, kept = 0;                        // a bit per group
            for (int n = 0; n < g.kept; ++n) {
                last = warp_max(a);
                if (last == 0) break;
                const int first = (__ffs(__ballot_sync(0xffffffffu, a == last)) - 1) >> p.group_shift;
                kept |= 1u << first;
                if (first == mine) a = 0;
            }
            if constexpr (kScored) {
                const uint32_t next = warp_max(a);              // the best that was left
                if (last != 0 && next != 0) unsure = !(value_of(last) - value_of(next) > 6.f * slack + 2.f * kUnit * fabsf(value_of(last)));
            }
            #pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (!(kept >> (p.side_by_side ? mine & 31 : (lane * VPL + i) / p.group_size & 31) & 1u)) key[i] = 0;
        }
        Choice c{-1, -INFINITY};
        if (!unsure) {
            uint32_t best = 0, last = 0;
            #pragma unroll
            for (int i = 0; i < VPL; ++i) best = max(best, key[i]);
            for (int j = 0; j < k; ++j) {
                const uint32_t now = warp_max(best);
                if (now == 0) { last = 0; break; }
                if constexpr (kScored) {
                    if (j > 0) unsure = unsure || !(value_of(last) - value_of(now) > 2.f * slack);
                    last = now;
                }
                // the lowest index is the first lane's first; every lane looks for its own, without branches
                const int from = __ffs(__ballot_sync(0xffffffffu, best == now)) - 1;
                uint32_t same = 0;
                #pragma unroll
                for (int i = 0; i < VPL; ++i) same |= (uint32_t)(key[i] == now) << i;
                const int own = __ffs(same) - 1, at = __shfl_sync(0xffffffffu, lane * VPL + own, from);
                best = 0;
                #pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    if (lane == from && i == own) key[i] = 0;
                    best = max(best, key[i]);
                }
                if (lane == j) c.pick = at;
            }
            if constexpr (kScored) {
                const uint32_t next = warp_max(best);
                if (last != 0 && next != 0) unsure = unsure || !(value_of(last) - value_of(next) > 2.f * slack);
            }
        }
        if (kScored && unsure) {
            if constexpr (kScored) {
                c = choose_exact<T, VPL>(g, t0 + t);
                if (c.pick == kOpen) { open |= 1u << (t / kWarps); continue; }
            }
        } else if (c.pick >= 0) c.logit = fminf(to_f32(static_cast<const T*>(g.logits)[(t0 + t) * g.stride + c.pick]), FLT_MAX);
        finish_token(g, t0 + t, c, top, sum, plan ? chosen : nullptr, words, t);
    }
    if constexpr (kScored) {
        for (; open != 0; open &= open - 1) {
            const int t = warp + (__ffs(open) - 1) * kWarps;
            choose_by_pairs<T>(g, t0 + t, plan ? chosen : nullptr, words, t);
        }
    }
    if (plan) note_block(g, chosen, t0, n_tok, words, counts);
}

// The same for many tokens, by logits alone and without groups: kShare threads side by side take a token, every fourth 16 bytes of its logits each, and
// keep the best kList experts of theirs in order; then the best of the four lists' heads is taken, top_k times, thread j % kShare has choice j.
// (A warp for each token: 600 instructions to a token; here 2 to 5 per expert and place of the list, for 8 of them.  A thread for each token by
// itself: one chain of the same length for all 128 experts, 110 threads to an SM.)
template <typename T> struct Entry;         // a key and its index in one word where the type has 16 bits: the larger, the earlier
template <> struct Entry<float> { uint32_t key; int index; };
template <typename T> struct Entry { uint32_t both; };
// Into the list, behind what is not smaller (indices only go up).
__device__ __forceinline__ void insert(Entry<float> (&list)[kList], const Entry<float>& x)
{
    bool before[kList];                                         // x's place is before this one, or this one
    #pragma unroll
    for (int j = 0; j < kList; ++j) before[j] = x.key > list[j].key;
    #pragma unroll
    for (int j = kList - 1; j >= 0; --j) {
        const Entry<float> in = j > 0 && before[j > 0 ? j - 1 : 0] ? list[j > 0 ? j - 1 : 0] : x;
        if (before[j]) list[j] = in;
    }
}
template <typename T>
__device__ __forceinline__ void insert(Entry<T> (&list)[kList], Entry<T> x)
{
    #pragma unroll
    for (int j = 0; j < kList; ++j) {
        const uint32_t high = max(list[j].both, x.both);
        x.both = min(list[j].both, x.both);
        list[j].both = high;
    }
}
template <typename T>
__device__ __forceinline__ Entry<T> entry_of(T logit, int index)
{
    const float v = to_f32(logit);
    const uint32_t key = v > -INFINITY ? key_of(sizeof(T) == 4 ? fminf(v, FLT_MAX) : v) : 0u;
    if constexpr (sizeof(T) == 4) return Entry<T>{key, index};
    else if constexpr (std::is_same<T, __half>::value) {
        const uint32_t u = __half_as_ushort(__float2half_rn(v + 0.f));
        return Entry<T>{key == 0 ? 0u : (u >> 15 ? ~u & 0xffffu : u | 0x8000u) << 16 | (uint32_t)(0xffff - index)};
    } else return Entry<T>{key == 0 ? 0u : key >> 16 << 16 | (uint32_t)(0xffff - index)};
}
__device__ __forceinline__ int index_of(const Entry<float>& e) { return e.key != 0 ? e.index : -1; }
template <typename T> __device__ __forceinline__ int index_of(const Entry<T>& e) { return e.both != 0 ? 0xffff - (int)(e.both & 0xffffu) : -1; }

// The best of the heads of the lists of kShare threads, which its thread takes off its list.
__device__ __forceinline__ Entry<float> take_best(Entry<float> (&list)[kList])
{
    uint32_t key = list[0].key;
    #pragma unroll
    for (int d = 1; d < kShare; d *= 2) key = max(key, __shfl_xor_sync(0xffffffffu, key, d));
    int at = list[0].key == key ? list[0].index : 0x7fffffff;
    const int own = at;
    #pragma unroll
    for (int d = 1; d < kShare; d *= 2) at = min(at, __shfl_xor_sync(0xffffffffu, at, d));
    if (key != 0 && own == at) {
        #pragma unroll
        for (int j = 0; j + 1 < kList; ++j) list[j] = list[j + 1];
        list[kList - 1] = Entry<float>{};
    }
    return Entry<float>{key, at};
}
template <typename T>
__device__ __forceinline__ Entry<T> take_best(Entry<T> (&list)[kList])
{
    uint32_t both = list[0].both;
    #pragma unroll
    for (int d = 1; d < kShare; d *= 2) both = max(both, __shfl_xor_sync(0xffffffffu, both, d));
    if (list[0].both == both) {                                 // (one thread, or nobody has any)
        #pragma unroll
        for (int j = 0; j + 1 < kList; ++j) list[j] = list[j + 1];
        list[kList - 1] = Entry<T>{};
    }
    return Entry<T>{both};
}

template <typename T>
__global__ void __launch_bounds__(kListThreads)
route_list_kernel(const __grid_constant__ RouteArgs g, int* counts)
{
    extern __shared__ uint32_t chosen[];
    constexpr int words = kListTokens / 32, kVec = 16 / (int)sizeof(T), kAhead = 4, kOwn = kList / kShare;
    const int64_t t0 = (int64_t)blockIdx.x * kListTokens;
    const int token = threadIdx.x / kShare, q = threadIdx.x % kShare;
    const int n_tok = g.T - t0 < kListTokens ? (int)(g.T - t0) : kListTokens, k = g.top_k;
    const int64_t t = t0 + (token < n_tok ? token : 0);         // (whoever has no token does another's, and writes nothing)
    const bool plan = g.start != nullptr;
    if (plan) {
        for (int i = threadIdx.x; i < g.E * words; i += kListThreads) chosen[i] = 0;
        __syncthreads();
    }
    tc::pdl_wait();
    const T* row = static_cast<const T*>(g.logits) + t * g.stride;
    Entry<T> list[kList];
    #pragma unroll
    for (int j = 0; j < kList; ++j) list[j] = Entry<T>{};
    const int vecs = (reinterpret_cast<uintptr_t>(row) & 15) == 0 ? g.E / kVec : 0;
    #pragma unroll 1
    for (int v0 = q; v0 < vecs; v0 += kShare * kAhead) {
        uint4 u[kAhead];
        #pragma unroll
        for (int i = 0; i < kAhead; ++i) u[i] = reinterpret_cast<const uint4*>(row)[v0 + i * kShare < vecs ? v0 + i * kShare : 0];
        #pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int v = v0 + i * kShare;
            if (v >= vecs) break;
            const T* x = reinterpret_cast<const T*>(&u[i]);
            #pragma unroll
            for (int j = 0; j < kVec; ++j) insert(list, entry_of(x[j], v * kVec + j));
        }
    }
    #pragma unroll 1
    for (int e0 = vecs * kVec + q; e0 < g.E; e0 += kShare * kAhead) {
        T x[kAhead];
        #pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = row[e0 + i * kShare < g.E ? e0 + i * kShare : 0];
        #pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (e0 + i * kShare < g.E) insert(list, entry_of(x[i], e0 + i * kShare));
    }
    __syncwarp();
    int pick[kOwn], first = -1;
    #pragma unroll
    for (int j = 0; j < kList; ++j) {
        const int at = index_of(take_best(list));
        if (j == 0) first = at;
        if (j % kShare == q) pick[j / kShare] = j < k ? at : -1;
    }
    const float best = first >= 0 ? fminf(to_f32(row[first]), FLT_MAX) : 0.f;
    auto shared_sum = [](float x) {
        #pragma unroll
        for (int d = 1; d < kShare; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
        return x;
    };
    float sum = 0.f, w[kOwn];
    if (g.score == RTN_SCORE_SOFTMAX && !g.renormalise) {
        #pragma unroll 4
        for (int e = q; e < g.E; e += kShare) {
            const float v = to_f32(row[e]);
            sum += v > -INFINITY ? __expf(fminf(v, FLT_MAX) - best) : 0.f;
        }
        sum = shared_sum(sum);
    }
    #pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        w[i] = 0.f;
        if (pick[i] < 0) continue;
        const float x = fminf(to_f32(row[pick[i]]), FLT_MAX);
        if (g.score == RTN_SCORE_SOFTMAX) w[i] = expf(x - best);
        else if (g.renormalise) w[i] = expf(fminf(x, 0.f) - fminf(best, 0.f)) / (1.f + expf(-fabsf(x)));
        else w[i] = 1.f / (1.f + expf(-x));
    }
    if (g.renormalise) {
        #pragma unroll
        for (int i = 0; i < kOwn; ++i) sum += w[i];
        sum = shared_sum(sum);
    } else if (g.score == RTN_SCORE_SIGMOID) sum = 1.f;
    #pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int j = i * kShare + q;
        if (j >= k || token >= n_tok) continue;
        g.experts[t * k + j] = pick[i];
        g.weights[t * k + j] = pick[i] >= 0 ? w[i] / sum * g.scale : 0.f;
        if (plan && pick[i] >= 0) atomicOr(&chosen[pick[i] * words + token / 32], 1u << (token & 31));
    }
    if (plan) note_block(g, chosen, t0, n_tok, words, counts);
}

// One expert's counts of all blocks as sums of those before; the total goes behind the last block's.
__global__ void __launch_bounds__(256)
route_scan_kernel(int E, int* counts, int64_t blocks)
{
    __shared__ int part[8];
    const int e = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    tc::pdl_wait();
    int before = 0;
    for (int64_t b0 = 0; b0 < blocks; b0 += 256) {
        const int64_t b = b0 + threadIdx.x;
        const int c = b < blocks ? counts[b * E + e] : 0;
        int x = c;
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) part[warp] = x;
        __syncthreads();
        int own = 0, all = 0;
        #pragma unroll
        for (int i = 0; i < 8; ++i) { own += i < warp ? part[i] : 0; all += part[i]; }
        if (b < blocks) counts[b * E + e] = before + own + x - c;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) counts[blocks * E + e] = before;
}

// scanned: counts are route_scan_kernel's.
__global__ void __launch_bounds__(kThreads)
route_plan_kernel(const RouteArgs g, const int* counts, int64_t blocks, int tokens, bool scanned)
{
    extern __shared__ int sums[];                               // total, before, start: [E + 1] each
    int *total = sums, *before = sums + g.E + 1, *start = before + g.E + 1;
    for (int e = threadIdx.x; e < g.E; e += kThreads) total[e] = before[e] = 0;
    tc::pdl_wait();
    __syncthreads();
    if (scanned) {
        for (int e = threadIdx.x; e < g.E; e += kThreads) { total[e] = counts[blocks * g.E + e]; before[e] = counts[(int64_t)blockIdx.x * g.E + e]; }
    } else {
        const int parts = g.E < kThreads ? kThreads / g.E : 1;
        for (int i = threadIdx.x; i < g.E * parts; i += kThreads) {
            const int e = i % g.E, p = i / g.E;
            int a = 0, b = 0;
            #pragma unroll 16
            for (int j = p; j < (int)blocks; j += parts) {
                const int c = counts[(int64_t)j * g.E + e];
                a += c;
                b += j < (int)blockIdx.x ? c : 0;
            }
            atomicAdd(&total[e], a);
            atomicAdd(&before[e], b);
        }
    }
    __syncthreads();
    if (threadIdx.x < 32) scan_counts(total, start, g.E, threadIdx.x);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= g.E; e += kThreads) g.start[e] = start[e];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int k = g.top_k, n = (int)((g.T - t0 < tokens ? g.T - t0 : tokens) * k);
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int e = g.experts[t0 * k + i];
        if (e < 0) continue;
        const int at = g.place[t0 * k + i] + start[e] + before[e];
        g.place[t0 * k + i] = at;
        g.tokens[at] = (int)(t0 + i / k);
    }
}

template <typename T, int VPL>
cudaError_t launch_choose(const RouteArgs& g, RoutePlan p, int* counts, unsigned blocks, cudaStream_t s)
{
    p.group_size = g.E / g.groups;
    const int lanes = p.group_size / VPL;
    p.side_by_side = p.group_size % VPL == 0 && (lanes & (lanes - 1)) == 0;
    p.group_shift = 0;
    while (p.side_by_side && 1 << p.group_shift < lanes) ++p.group_shift;
    const size_t smem = g.start != nullptr ? (size_t)g.E * ((p.tokens + 31) / 32) * 4 + 2 * (g.E + 1) * 4 : 0;
    // scores have to be computed where a bias or a sum of them is compared
    const bool scored = g.bias != nullptr || (g.groups > 1 && g.group_top > 1);
    return launch_pdl(scored ? route_choose_kernel<T, VPL, true> : route_choose_kernel<T, VPL, false>, dim3(blocks), dim3(kThreads), smem, s, g, p, counts);
}

}  // namespace

cudaError_t launch_route_experts(const RouteArgs& g, cudaStream_t s)
{
    if (g.T == 0) return cudaMemsetAsync(g.start, 0, (size_t)(g.E + 1) * sizeof(int32_t), s);
    // A token to each warp while there are few (a token's chain is what counts), more with more, so that about two blocks to an SM hold them
    // Lists from 4096 tokens on (in a graph on one B200, all kernels, us, lists and warps): 8 of 128 experts, bf16: 2048 tokens 10.6 and 9.2, 4096 10.6 and
    // 11.1, 16384 13.2 and 22.8, 65536 31.6 and 70.2; 8 of 256, fp32: 2048 17.0 and 11.6, 4096 16.6 and 16.3, 16384 22.1 and 34.6.  Eight
    // threads to a token, 64 tokens to a block: 12.7 at 16384 and 35.6 at 65536; four and 128: 12.8 and 30.8, but 12.3 for 10.9 at 8192.
    const bool listed = g.T >= kListFrom && g.top_k <= kList && g.groups == 1 && g.bias == nullptr;
    RoutePlan p{kWarps, 0, 0, false};
    if (listed) p.tokens = kListTokens;
    else while (p.tokens < kMaxTokens && g.T > (int64_t)2 * device_sm_count() * p.tokens) p.tokens *= 2;
    const int64_t blocks = (g.T + p.tokens - 1) / p.tokens;
    const bool scanned = blocks > kScanBlocks;
    void* counts = nullptr;
    if (g.start != nullptr && blocks > 1) {
        const cudaError_t e = scratch_alloc(&counts, (size_t)(blocks + 1) * g.E * sizeof(int), s);
        if (e != cudaSuccess) return e;
    }
    int* c = static_cast<int*>(counts);
    cudaError_t e = with_dtype(g.dtype, [&](auto t) {
        using T = decltype(t);
        if (listed) {
            const size_t smem = g.start != nullptr ? (size_t)g.E * (kListTokens / 32) * 4 + 2 * (g.E + 1) * 4 : 0;
            return launch_pdl(route_list_kernel<T>, dim3((unsigned)blocks), dim3(kListThreads), smem, s, g, c);
        }
        if (g.E <= 32) return launch_choose<T, 1>(g, p, c, (unsigned)blocks, s);
        if (g.E <= 64) return launch_choose<T, 2>(g, p, c, (unsigned)blocks, s);
        if (g.E <= 128) return launch_choose<T, 4>(g, p, c, (unsigned)blocks, s);
        if (g.E <= 256) return launch_choose<T, 8>(g, p, c, (unsigned)blocks, s);
        if (g.E <= 512) return launch_choose<T, 16>(g, p, c, (unsigned)blocks, s);
        return launch_choose<T, 32>(g, p, c, (unsigned)blocks, s);
    });
    if (e == cudaSuccess && counts != nullptr) {
        const size_t smem = (size_t)3 * (g.E + 1) * sizeof(int);
        if (scanned) {
            e = launch_pdl(route_scan_kernel, dim3((unsigned)g.E), dim3(256), 0, s, g.E, c, blocks);
            // (it reads what the kernel before the last one has written, which the last one has waited for)
            if (e == cudaSuccess) e = launch_pdl(route_plan_kernel, dim3((unsigned)blocks), dim3(kThreads), smem, s, g, (const int*)counts, blocks, p.tokens, true);
        } else {
            e = launch_pdl(route_plan_kernel, dim3((unsigned)blocks), dim3(kThreads), smem, s, g, (const int*)counts, blocks, p.tokens, false);
        }
    }
    if (counts != nullptr) {
        const cudaError_t e2 = cudaFreeAsync(counts, s);
        if (e == cudaSuccess) e = e2;
    }
    return e;
}

}  // namespace rtn
