// The norms after one block and before the next, with the block's gate, its residual and the experts' weighted sum, and the codes of the
// result: a CTA per token, the token's values in registers between the passes (what of them does not fit is with the launcher's rule).
//
// Bound: HBM, every input and output once.
//
// Codes are those of the exact value.  Beside each value runs a bound on its rounding error in units of u = 2^-24 (to first order):
//   y = sum_j w_j x_j, one rounding per term           E_y <= the sum of the partial sums' magnitudes   (0 without experts)
//   1/sqrt(mean + eps) of a sum of squares over a tree  relative: (half of the tree's depth) + |E| / |.| (of the vector norms)
// and so on through gate, scale and residual.  A value nearer to a threshold than its bound, or one that is not finite, makes the CTA work
// the token's codes out again in double; of tokens of 2048 normal values about one in a hundred.  That pass takes 10 us, which is what the last of a
// launch's rows that needs it adds (with thresholds that nothing is near, the 124 us below are 112).  A value that equals its threshold is always too near:
// rows without a norm in 16 bits lie on values of their type, and with a threshold that is one of these nearly every token is worked out
// again (8192 x 2048, bf16 135 us, with a threshold between two of them 37).
// Measured (one B200): 8192 tokens of 2048, bf16, 8 experts' rows each, both norms, codes 124 us (407 MB: 62 at the copy rate; the rest is issue slots, some
// 1200 instructions per 256 values, at half the occupancy), values in place of codes 84 us; without experts 83 and 49 us; one token of 2048, 4 rows, codes 3.4 us
// in a graph; 48 of 4096, gated 3.4 us; 1111 of 5003, fp32, one value to an access 30.3 us.
#include "rtn_internal.cuh"
#include "rtn_epilogue.cuh"
#include "rtn_tcgen05.cuh"

namespace rtn {

namespace {

constexpr float kUnit = 5.9604644775390625e-8f;                // 2^-24
constexpr int kMaxWarps = 32;

// EV adjacent elements in accesses of up to 16 bytes (the launcher saw to the alignment).  `Held` is what they are until they are looked at, so that
// many are on their way at a time.
template <int kBytes> struct Word { uint4 u[kBytes / 16]; };
template <> struct Word<2> { unsigned short u; };
template <> struct Word<4> { uint32_t u; };
template <> struct Word<8> { uint2 u; };
template <typename T, int EV> using Held = Word<EV * (int)sizeof(T)>;

template <typename T, int EV>
__device__ __forceinline__ Held<T, EV> ask(const T* row, int at)
{
    Held<T, EV> h;
    if constexpr (EV * sizeof(T) > 16) {
        #pragma unroll
        for (int i = 0; i < EV * (int)sizeof(T) / 16; ++i) h.u[i] = reinterpret_cast<const uint4*>(row + at)[i];
    } else h = *reinterpret_cast<const Held<T, EV>*>(row + at);
    return h;
}
template <typename T, int EV>
__device__ __forceinline__ void take(const Held<T, EV>& h, bool ok, float (&f)[EV])       // zeros where not ok
{
    const T* e = reinterpret_cast<const T*>(&h);
    #pragma unroll
    for (int i = 0; i < EV; ++i) f[i] = ok ? to_f32(e[i]) : 0.f;
}
template <typename T, int EV>
__device__ __forceinline__ void store_values(T* row, int at, const float (&f)[EV])
{
    alignas(16) T e[EV];
    #pragma unroll
    for (int i = 0; i < EV; ++i) e[i] = from_f32<T>(f[i]);
    if constexpr (EV * sizeof(T) > 16) {
        #pragma unroll
        for (int i = 0; i < EV * (int)sizeof(T) / 16; ++i) reinterpret_cast<uint4*>(row + at)[i] = reinterpret_cast<const uint4*>(e)[i];
    } else *reinterpret_cast<Held<T, EV>*>(row + at) = *reinterpret_cast<const Held<T, EV>*>(e);
}
template <int EV>
__device__ __forceinline__ void load_params(const float* p, int at, float (&f)[EV])
{
    take<float, EV>(ask<float, EV>(p, at), true, f);
}

// Sums of a pair over the block; every thread has them.
template <typename F>
__device__ __forceinline__ void block_sums(F& a, F& b, F* red)
{
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, d); b += __shfl_xor_sync(0xffffffffu, b, d); }
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (warps == 1) return;
    __syncthreads();                                           // (the last sums have been read)
    if (lane == 0) { red[2 * (threadIdx.x >> 5)] = a; red[2 * (threadIdx.x >> 5) + 1] = b; }
    __syncthreads();
    a = lane < warps ? red[2 * lane] : (F)0;
    b = lane < warps ? red[2 * lane + 1] : (F)0;
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, d); b += __shfl_xor_sync(0xffffffffu, b, d); }
}

// By the approximate exponential (4 units of 2^-24) and reciprocal (2).  Rounded, the exponent is off by |z| units, its constant by another 0.22 |z|, so the
// logistic function is within (1.25 |z| + 4) (1 - s) + 3 units, relative: below 8 for z >= 0, but growing with how far a gate is closed.  Below -87
// it leaves fp32's normal range and is 0.
constexpr float kShut = -746.f;             // the logistic function is 0 in double, too
__device__ __forceinline__ float gate_of(float z, int kind)
{
    if (kind == RTN_GATE_LINEAR) return z;
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
    return kind == RTN_GATE_SIGMOID ? s : z * s;
}

// Square root of a quotient, for bounds only.
__device__ __forceinline__ float root_of_ratio(float a, float b)
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(__fdividef(a, b)));
    return r;
}
// Units of a root's error: roundings of the sum of squares `ss`, per thread and over two trees, of the mean and of the root (approximate: two units in the last
// place of 2^-23), and the values' own errors, whose squares add up to `sm`.  No bound where squares leave fp32: what
// falls below its normal range is less than 2^-149 each, nothing beside a mean (with eps: `square`) of 1e-30; above 2^126 the quotient is 0.  And none
// where the values' errors are more than a 64th of them (sums that cancel): bounds are to first order.
template <int NV, int EV>
__device__ __forceinline__ float root_units(float square, float ss, float sm)
{
    const float units = 0.5f * (NV * EV + 10) + 6.f + (ss > 0.f ? root_of_ratio(sm, ss) : 0.f);
    return square > 1e-30f && ss < 8e37f && units < 262144.f ? units : INFINITY;
}

// h and n of token t.  slack receives the bound on n's error, where kTrack asks for it.  Loads are not in branches (a value behind the row's end is
// read from its beginning and put to zero): the compiler waited for one after the other there.
template <typename TB, typename TS, int EV, int NV, bool kTrack>
__device__ __forceinline__ void norm_row(const NormArgs& g, int64_t t, float* red, float (&h)[NV][EV], float (&n)[NV][EV], float (&slack)[NV][EV])
{
    const int W = g.W, step = blockDim.x * EV, first = threadIdx.x * EV;
    const float mean = 1.f / (float)W;
    float zero = 0.f, ss = 0.f, sm = 0.f, closed = 0.f;
    int at[NV];                                                 // a value's column, or 0 behind the row's end
    bool in[NV];
    #pragma unroll
    for (int v = 0; v < NV; ++v) { in[v] = first + v * step < W; at[v] = in[v] ? first + v * step : 0; }
    Held<TS, EV> res[NV];
    if (g.residual != nullptr) {
        #pragma unroll
        for (int v = 0; v < NV; ++v) res[v] = ask<TS, EV>(static_cast<const TS*>(g.residual) + t * g.residual_stride, at[v]);
    }
    // y in h, the sum of its partial sums' magnitudes in slack
    #pragma unroll
    for (int v = 0; v < NV; ++v)
        #pragma unroll
        for (int i = 0; i < EV; ++i) h[v][i] = slack[v][i] = 0.f;
    if (g.place != nullptr && g.R == 0) {                       // no rows to read, not even for a place that is out of range
        bool bad = false;
        for (int j = 0; j < g.k; ++j) bad = bad || g.place[t * g.k + j] >= 0;
        #pragma unroll
        for (int v = 0; v < NV; ++v)
            #pragma unroll
            for (int i = 0; i < EV; ++i) h[v][i] = bad ? __int_as_float(0x7fffffff) : 0.f;
    } else if (g.place != nullptr) {
        constexpr int kAhead = NV * EV <= 8 ? 4 : 1;            // rows on their way
        #pragma unroll 1
        for (int j0 = 0; j0 < g.k; j0 += kAhead) {
            Held<TB, EV> x[kAhead][NV];
            float w[kAhead];
            bool ok[kAhead];
            #pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int j = j0 + i < g.k ? j0 + i : 0;
                const int64_t row = g.place[t * g.k + j];
                w[i] = g.weights != nullptr ? g.weights[t * g.k + j] : 1.f;
                ok[i] = j0 + i < g.k && row >= 0 && row < g.R;
                if (!ok[i]) w[i] = j0 + i < g.k && row >= g.R ? __int_as_float(0x7fffffff) : 0.f;
                #pragma unroll
                for (int v = 0; v < NV; ++v) x[i][v] = ask<TB, EV>(static_cast<const TB*>(g.branch) + (ok[i] ? row : 0) * g.branch_stride, at[v]);
            }
            #pragma unroll
            for (int i = 0; i < kAhead; ++i)
                #pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float f[EV];
                    take<TB, EV>(x[i][v], ok[i], f);
                    if constexpr (EV > 1) {                                      // (two products to an instruction)
                        #pragma unroll
                        for (int e = 0; e < EV; e += 2)
                            take_pair(fma_pair(make_pair(w[i], w[i]), make_pair(f[e], f[e + 1]), make_pair(h[v][e], h[v][e + 1])), h[v][e], h[v][e + 1]);
                    } else h[v][0] = fmaf(w[i], f[0], h[v][0]);
                    if constexpr (kTrack) {
                        #pragma unroll
                        for (int e = 0; e < EV; ++e) slack[v][e] += fabsf(h[v][e]);
                    }
                }
        }
        #pragma unroll
        for (int v = 0; v < NV; ++v)
            if (!in[v]) {
                #pragma unroll
                for (int e = 0; e < EV; ++e) h[v][e] = slack[v][e] = 0.f;
            }
    } else if (g.branch != nullptr) {
        Held<TB, EV> x[NV];
        #pragma unroll
        for (int v = 0; v < NV; ++v) x[v] = ask<TB, EV>(static_cast<const TB*>(g.branch) + t * g.branch_stride, at[v]);
        #pragma unroll
        for (int v = 0; v < NV; ++v) take<TB, EV>(x[v], in[v], h[v]);
    }
    // what y is multiplied with, apart from its norm
    float f[NV][EV];
    float units = g.post_weight != nullptr ? 2.f : 0.f;         // roundings of the factor and its product
    #pragma unroll
    for (int v = 0; v < NV; ++v)
        #pragma unroll
        for (int i = 0; i < EV; ++i) f[v][i] = 1.f;
    if (g.gate != nullptr) {
        Held<TB, EV> z[NV];
        #pragma unroll
        for (int v = 0; v < NV; ++v) z[v] = ask<TB, EV>(static_cast<const TB*>(g.gate) + t * g.gate_stride, at[v]);
        #pragma unroll
        for (int v = 0; v < NV; ++v) {
            take<TB, EV>(z[v], true, f[v]);
            if constexpr (kTrack) {
                if (g.gate_kind != RTN_GATE_LINEAR) {
                    #pragma unroll
                    for (int i = 0; i < EV; ++i) closed = fmaxf(closed, f[v][i] > kShut ? -f[v][i] : 0.f);
                }
            }
            #pragma unroll
            for (int i = 0; i < EV; ++i) f[v][i] = gate_of(f[v][i], g.gate_kind);
        }
        // (one bound for all of a thread's values, by its most closed gate; none where that is 0 in fp32 only)
        units += closed < 87.f ? fmaf(1.25f, closed, 12.f) : INFINITY;
    }
    if (g.scale != nullptr) {
        units += 1.f;
        if (g.n_scale == 1) {
            #pragma unroll
            for (int v = 0; v < NV; ++v)
                #pragma unroll
                for (int i = 0; i < EV; ++i) f[v][i] *= g.scale[0];
        } else {
            #pragma unroll
            for (int v = 0; v < NV; ++v) {
                float p[EV];
                load_params<EV>(g.scale, at[v], p);
                #pragma unroll
                for (int i = 0; i < EV; ++i) f[v][i] *= p[i];
            }
        }
    }
    float post_units = 0.f;
    if (g.post_weight != nullptr) {
        #pragma unroll
        for (int v = 0; v < NV; ++v) {
            float p[EV];
            load_params<EV>(g.post_weight, at[v], p);
            #pragma unroll
            for (int i = 0; i < EV; ++i) {
                f[v][i] *= p[i];
                ss = fmaf(h[v][i], h[v][i], ss);
                if constexpr (kTrack) sm = fmaf(slack[v][i], slack[v][i], sm);
            }
        }
        block_sums(ss, kTrack ? sm : zero, red);
        const float square = fmaf(ss, mean, g.eps), post = rsqrtf(square);
        if constexpr (kTrack) post_units = root_units<NV, EV>(square, ss, sm) + 2.f;
        #pragma unroll
        for (int v = 0; v < NV; ++v)
            #pragma unroll
            for (int i = 0; i < EV; ++i) f[v][i] *= post;
        ss = sm = 0.f;
    }
    const float y_units = post_units + units;
    #pragma unroll
    for (int v = 0; v < NV; ++v) {
        float r[EV];
        #pragma unroll
        for (int i = 0; i < EV; ++i) r[i] = 0.f;
        if (g.residual != nullptr) take<TS, EV>(res[v], in[v], r);
        #pragma unroll
        for (int i = 0; i < EV; ++i) {
            const float y = h[v][i], m = slack[v][i], q = in[v] ? f[v][i] : 0.f;       // (behind the row's end y, its terms and r are zeros)
            h[v][i] = fmaf(q, y, r[i]);
            if constexpr (kTrack) {
                slack[v][i] = fmaf(fabsf(q), fmaf(y_units, fabsf(y), m), fabsf(h[v][i]));
                sm = fmaf(slack[v][i], slack[v][i], sm);
            }
            ss = fmaf(h[v][i], h[v][i], ss);
        }
    }
    float pre_units = 0.f;
    if (g.norm_weight != nullptr) {
        float p[NV][EV];
        #pragma unroll
        for (int v = 0; v < NV; ++v) load_params<EV>(g.norm_weight, at[v], p[v]);
        block_sums(ss, kTrack ? sm : zero, red);
        const float square = fmaf(ss, mean, g.eps), pre = rsqrtf(square);
        if constexpr (kTrack) pre_units = root_units<NV, EV>(square, ss, sm) + 4.f;
        #pragma unroll
        for (int v = 0; v < NV; ++v)
            #pragma unroll
            for (int i = 0; i < EV; ++i) {
                const float q = pre * p[v][i];
                n[v][i] = q * h[v][i];
                if constexpr (kTrack) slack[v][i] = fabsf(q) * fmaf(pre_units, fabsf(h[v][i]), slack[v][i]);
            }
    } else {
        #pragma unroll
        for (int v = 0; v < NV; ++v)
            #pragma unroll
            for (int i = 0; i < EV; ++i) n[v][i] = h[v][i];
    }
}

// One bit per value: above the upper threshold, below the lower one.  True: some value is within its bound of a threshold, or not finite.
template <int EV, int NV>
__device__ __forceinline__ bool code_row(const NormArgs& g, const float (&n)[NV][EV], const float (&slack)[NV][EV], uint32_t& up, uint32_t& down)
{
    up = down = 0;
    bool near = false;
    #pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = threadIdx.x * EV + v * blockDim.x * EV;
        if (c >= g.W) continue;
        float lo[EV], hi[EV];
        if (g.n_thr == 1) {
            #pragma unroll
            for (int i = 0; i < EV; ++i) { lo[i] = g.t_lo[0]; hi[i] = g.t_hi[0]; }
        } else {
            load_params<EV>(g.t_lo, c, lo);
            load_params<EV>(g.t_hi, c, hi);
        }
        #pragma unroll
        for (int i = 0; i < EV; ++i) {
            const float x = n[v][i];
            const bool a = x > hi[i], b = !a && x < lo[i];
            up |= (uint32_t)a << (v * EV + i);
            down |= (uint32_t)b << (v * EV + i);
            const float d = fminf(fabsf(x - lo[i]), fabsf(x - hi[i]));        // (a difference that small is exact but for its own rounding)
            near = near || !(d > fmaf(1.25f * kUnit, slack[v][i], 1e-37f));          // (of a NaN, and of what over- or underflowed)
        }
    }
    return near;
}

// The codes of one token in double: thread by thread the columns threadIdx.x, threadIdx.x + blockDim.x, ..., kTogether of them with their loads on
// their way together (a row's turn is some ten latencies; one column and one kind of load after the other took four times as long, and the last of
// a launch's rows that needed it was what the launch waited for).
constexpr int kExactEach = 16, kTogether = 4;                   // columns of a thread at most
template <typename TB, typename TS>
static __device__ __noinline__ int exact_codes(const NormArgs& g, int64_t t, double* red, uint8_t* row)
{
    const int W = g.W, step = blockDim.x;
    double h[kExactEach], post = 1.0, pre = 1.0, none = 0.0, ss = 0.0;
    const TB* branch = static_cast<const TB*>(g.branch);
    #pragma unroll 1
    for (int i0 = 0, c0 = threadIdx.x; c0 < W; i0 += kTogether, c0 += kTogether * step) {
        double y[kTogether];
        #pragma unroll
        for (int u = 0; u < kTogether; ++u) y[u] = 0.0;
        if (g.place != nullptr && g.R == 0) {
            bool bad = false;
            for (int j = 0; j < g.k; ++j) bad = bad || g.place[t * g.k + j] >= 0;
            #pragma unroll
            for (int u = 0; u < kTogether; ++u) y[u] = bad ? __longlong_as_double(0x7fffffffffffffffll) : 0.0;
        } else if (g.place != nullptr) {
            #pragma unroll 1
            for (int j0 = 0; j0 < g.k; j0 += 4) {
                TB x[4][kTogether];
                float w[4];
                bool ok[4];
                #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = j0 + i < g.k ? j0 + i : 0;
                    const int64_t r = g.place[t * g.k + j];
                    w[i] = g.weights != nullptr ? g.weights[t * g.k + j] : 1.f;
                    ok[i] = j0 + i < g.k && r >= 0;
                    if (ok[i] && r >= g.R) w[i] = __int_as_float(0x7fffffff);
                    const TB* from = branch + (ok[i] && r < g.R ? r : 0) * g.branch_stride;
                    #pragma unroll
                    for (int u = 0; u < kTogether; ++u) x[i][u] = from[c0 + u * step < W ? c0 + u * step : 0];
                }
                #pragma unroll
                for (int i = 0; i < 4; ++i)
                    #pragma unroll
                    for (int u = 0; u < kTogether; ++u)
                        if (ok[i]) y[u] = fma((double)w[i], (double)to_f32(x[i][u]), y[u]);
            }
        } else if (branch != nullptr) {
            TB x[kTogether];
            #pragma unroll
            for (int u = 0; u < kTogether; ++u) x[u] = branch[t * g.branch_stride + (c0 + u * step < W ? c0 + u * step : 0)];
            #pragma unroll
            for (int u = 0; u < kTogether; ++u) y[u] = (double)to_f32(x[u]);
        }
        #pragma unroll
        for (int u = 0; u < kTogether; ++u)
            if (c0 + u * step < W) { h[i0 + u] = y[u]; ss = fma(y[u], y[u], ss); }
    }
    if (g.post_weight != nullptr) {
        block_sums(ss, none, red);
        post = 1.0 / sqrt(ss / (double)W + (double)g.eps);
    }
    ss = none = 0.0;
    const TB* gate = static_cast<const TB*>(g.gate) + t * g.gate_stride;
    const TS* residual = static_cast<const TS*>(g.residual) + t * g.residual_stride;
    const double scale = g.scale != nullptr && g.n_scale == 1 ? (double)g.scale[0] : 1.0;
    #pragma unroll 1
    for (int i0 = 0, c0 = threadIdx.x; c0 < W; i0 += kTogether, c0 += kTogether * step) {
        float r[kTogether], z[kTogether], p[kTogether], q[kTogether];
        #pragma unroll
        for (int u = 0; u < kTogether; ++u) { r[u] = 0.f; z[u] = p[u] = q[u] = 1.f; }
        #pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int c = c0 + u * step < W ? c0 + u * step : 0;
            if (g.residual != nullptr) r[u] = to_f32(residual[c]);
            if (g.gate != nullptr) z[u] = to_f32(gate[c]);
            if (g.post_weight != nullptr) p[u] = g.post_weight[c];
            if (g.scale != nullptr && g.n_scale != 1) q[u] = g.scale[c];
        }
        #pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            if (c0 + u * step >= W) continue;
            double f = scale * (double)q[u] * (post * (double)p[u]);
            if (g.gate != nullptr) {
                if (g.gate_kind != RTN_GATE_SIGMOID) f *= (double)z[u];
                if (g.gate_kind != RTN_GATE_LINEAR) {
                    const double e = exp(-fabs((double)z[u]));                     // (of -z it would leave the range at 710)
                    f *= (z[u] < 0.f ? e : 1.0) / (1.0 + e);
                }
            }
            const double y = branch != nullptr || g.place != nullptr ? fma(f, h[i0 + u], (double)r[u]) : (double)r[u];
            h[i0 + u] = y;
            ss = fma(y, y, ss);
        }
    }
    if (g.norm_weight != nullptr) {
        block_sums(ss, none, red);
        pre = 1.0 / sqrt(ss / (double)W + (double)g.eps);
    }
    int sum = 0;
    const int width = (W + kBlockCodes - 1) / kBlockCodes * kBlockCodes, lane = threadIdx.x & 31;
    #pragma unroll 1
    for (int i0 = 0, c0 = threadIdx.x & ~31; c0 < width; i0 += kTogether, c0 += kTogether * step) {
        float p[kTogether], lo[kTogether], hi[kTogether];
        #pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int c = c0 + lane + u * step < W ? c0 + lane + u * step : 0, k = g.n_thr == 1 ? 0 : c;
            p[u] = 1.f;
            if (g.norm_weight != nullptr) p[u] = g.norm_weight[c];
            lo[u] = g.t_lo[k];
            hi[u] = g.t_hi[k];
        }
        #pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int first = c0 + u * step;
            if (first >= width) continue;
            bool up = false, down = false;
            if (first + lane < W) {
                const double n = h[i0 + u] * (pre * (double)p[u]);
                up = n > (double)hi[u];
                down = !up && n < (double)lo[u];
            }
            const uint32_t a = __ballot_sync(0xffffffffu, up), b = __ballot_sync(0xffffffffu, down);
            if (lane == 0) {
                uint32_t* at = reinterpret_cast<uint32_t*>(row + first / kBlockCodes * kBlockBytes + first % kBlockCodes / 8);
                at[0] = a | b;
                at[4] = a;
                sum += __popc(a) - __popc(b);
            }
        }
    }
    return sum;
}

// The low 16 bits, at the even places.
__device__ __forceinline__ uint32_t spread(uint32_t x)
{
    x &= 0xffffu;
    x = (x | x << 8) & 0x00ff00ffu;
    x = (x | x << 4) & 0x0f0f0f0fu;
    x = (x | x << 2) & 0x33333333u;
    return (x | x << 1) & 0x55555555u;
}

template <typename TB, typename TS, int EV, int NV, int kMaxThreads, bool kCodes>
__global__ void __launch_bounds__(kMaxThreads, kMaxThreads == 640 ? 2 : 1024 / kMaxThreads)
block_norm_kernel(const __grid_constant__ NormArgs g)
{
    __shared__ double red[2 * kMaxWarps];
    const int64_t t = blockIdx.x;
    tc::pdl_wait();
    float h[NV][EV], n[NV][EV], slack[NV][EV];
    norm_row<TB, TS, EV, NV, kCodes>(g, t, reinterpret_cast<float*>(red), h, n, slack);
    if constexpr (kCodes) {
        uint32_t up, down;
        const bool near = code_row<EV, NV>(g, n, slack, up, down);
        const int blocks = (g.W + kBlockCodes - 1) / kBlockCodes;
        uint8_t* row = g.out_packed + t * blocks * kBlockBytes;
        int own = __popc(up) - __popc(down);
        if (__syncthreads_or(near)) {
            own = exact_codes<TB, TS>(g, t, red, row);
        } else {
            #pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = threadIdx.x * EV + v * blockDim.x * EV;
                if constexpr (EV == 8) {
                    if (c < blocks * kBlockCodes) {
                        uint8_t* at = row + c / kBlockCodes * kBlockBytes + c % kBlockCodes / 8;
                        at[0] = (uint8_t)(up >> (v * 8) | down >> (v * 8));
                        at[16] = (uint8_t)(up >> (v * 8));
                    }
                } else {
                    // a warp's 32 EV values: EV words of each plane, the values of a lane side by side
                    uint32_t nz[EV], pos[EV];
                    #pragma unroll
                    for (int i = 0; i < EV; ++i) {
                        pos[i] = __ballot_sync(0xffffffffu, up >> (v * EV + i) & 1);
                        nz[i] = __ballot_sync(0xffffffffu, (up | down) >> (v * EV + i) & 1);
                    }
                    const int lane = threadIdx.x & 31, word = c - lane * EV + lane * 32;       // the word's first column, for lanes below EV
                    if (lane < EV && word < blocks * kBlockCodes) {
                        uint32_t a = nz[0], b = pos[0];
                        if constexpr (EV == 2) {
                            auto both = [&](uint32_t x, uint32_t y) { return spread(x >> (16 * lane)) | spread(y >> (16 * lane)) << 1; };
                            a = both(nz[0], nz[1]); b = both(pos[0], pos[1]);
                        }
                        uint32_t* at = reinterpret_cast<uint32_t*>(row + word / kBlockCodes * kBlockBytes + word % kBlockCodes / 8);
                        at[0] = a;
                        at[4] = b;
                    }
                }
            }
        }
        own = __reduce_add_sync(0xffffffffu, own);
        int* sums = reinterpret_cast<int*>(red);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = own;
        __syncthreads();
        if (threadIdx.x < 32) {
            own = __reduce_add_sync(0xffffffffu, (int)threadIdx.x < (int)(blockDim.x >> 5) ? sums[threadIdx.x] : 0);
            if (threadIdx.x == 0) g.out_sum[t] = own;
        }
    }
    #pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = threadIdx.x * EV + v * blockDim.x * EV;
        if (c >= g.W) continue;
        if (g.stream_out != nullptr) store_values<TS, EV>(static_cast<TS*>(g.stream_out) + t * g.stream_stride, c, h[v]);
        if (g.normed != nullptr) store_values<TB, EV>(static_cast<TB*>(g.normed) + t * g.normed_stride, c, n[v]);
    }
    if (g.place != nullptr && threadIdx.x < g.k && g.place[t * g.k + threadIdx.x] >= g.R) atomicOr(g.status, kStatusBadIndex);
}

template <typename TB, typename TS, int EV, int NV, int kMaxThreads>
cudaError_t launch_values(const NormArgs& g, cudaStream_t s)
{
    const int width = (g.W + kBlockCodes - 1) / kBlockCodes * kBlockCodes;         // (the padding of a packed row is written too)
    const int threads = ((width + EV * NV - 1) / (EV * NV) + 31) / 32 * 32;
    const bool coded = g.out_packed != nullptr;
    return launch_pdl(coded ? block_norm_kernel<TB, TS, EV, NV, kMaxThreads, true> : block_norm_kernel<TB, TS, EV, NV, kMaxThreads, false>, dim3((unsigned)g.T), dim3(threads), 0, s, g);
}

template <typename TB, typename TS>
cudaError_t launch_types(const NormArgs& g, cudaStream_t s)
{
    // Adjacent values that a thread may take at a time: eight or two where every row and parameter lets it, else one
    auto fits = [&](int ev) {
        auto ok = [&](const void* p, int64_t stride, size_t e) {
            const uintptr_t bytes = ev * e < 16 ? ev * e : 16;
            return p == nullptr || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && stride * (int64_t)e % (int64_t)bytes == 0);
        };
        return g.W % ev == 0 && ok(g.branch, g.branch_stride, sizeof(TB)) && ok(g.gate, g.gate_stride, sizeof(TB)) &&
               ok(g.normed, g.normed_stride, sizeof(TB)) && ok(g.residual, g.residual_stride, sizeof(TS)) &&
               ok(g.stream_out, g.stream_stride, sizeof(TS)) && ok(g.post_weight, 0, 4) && ok(g.norm_weight, 0, 4) &&
               (g.n_scale == 1 || ok(g.scale, 0, 4)) && (g.n_thr == 1 || (ok(g.t_lo, 0, 4) && ok(g.t_hi, 0, 4)));
    };
    // A thread has 8 values, and only above 5120 16 where they do not come eight to an access.  Eight to an access and without codes all of them stay in its
    // 56 to 64 registers (up to 8192 wide); in the other forms without codes up to 204 bytes a thread go to local memory, and the bounds beside the values
    // make that 120 to 152 bytes with codes, eight to an access, and 180 to 512 in the others (of -Xptxas -v).  Rows of up to 5120 values in one or two to an access, two blocks of up to
    // 640 threads to an SM, which leaves a thread 48 registers, instead of 16 values a thread, 1111 tokens, fp32, normed and codes: 5003 33.1 and 77.3 -> 32.7 and 63.6 us, 5002 33.9 and
    // 69.4 -> 29.7 and 58.2, 2500 16.4 and 40.8 -> 11.5 and 32.1.
    if (fits(8)) {
        if (g.W <= 2048) return launch_values<TB, TS, 8, 1, 256>(g, s);
        return g.W <= 8192 ? launch_values<TB, TS, 8, 1, 1024>(g, s) : launch_values<TB, TS, 8, 2, 1024>(g, s);
    }
    if (fits(2)) {
        if (g.W <= 2048) return launch_values<TB, TS, 2, 4, 256>(g, s);
        if (g.W <= 5120) return launch_values<TB, TS, 2, 4, 640>(g, s);
        return g.W <= 8192 ? launch_values<TB, TS, 2, 8, 512>(g, s) : launch_values<TB, TS, 2, 8, 1024>(g, s);
    }
    if (g.W <= 2048) return launch_values<TB, TS, 1, 8, 256>(g, s);
    if (g.W <= 5120) return launch_values<TB, TS, 1, 8, 640>(g, s);
    return g.W <= 8192 ? launch_values<TB, TS, 1, 16, 512>(g, s) : launch_values<TB, TS, 1, 16, 1024>(g, s);
}

}  // namespace

cudaError_t launch_block_norm(const NormArgs& g, cudaStream_t s)
{
    return with_dtype(g.dtype, [&](auto b) {
        return with_dtype(g.stream_dtype, [&](auto t) { return launch_types<decltype(b), decltype(t)>(g, s); });
    });
}

}  // namespace rtn
