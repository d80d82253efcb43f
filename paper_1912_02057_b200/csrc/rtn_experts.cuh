// Shared by the kernels of the experts' products: which rows a tile has, the epilogue and its codes.
#pragma once
#include "rtn_internal.cuh"
#include "rtn_epilogue.cuh"

namespace rtn {

cudaError_t launch_experts_tiles(const ExpertsArgs& g, cudaStream_t s);        // on the tensor cores
bool experts_tiles_supported(const ExpertsArgs& g);

#ifdef __CUDACC__

// Tile `index` of the experts' rows, each expert's in tiles of `height`: expert (-1: there are not so many tiles), first row and rows.
// A whole warp asks; a lane looks at one expert of 32 at a time.  An expert whose bounds do not fit has no rows.
struct RowTile { int e, row, rows; };
__device__ __forceinline__ RowTile find_tile(const int32_t* __restrict__ start, int E, int64_t R, int height, int index, unsigned* status)
{
    const int lane = threadIdx.x & 31;
    RowTile r{-1, 0, 0};
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
        const int e = e0 + lane;
        int s = 0, n = 0;
        if (e < E) {
            s = start[e];
            const int64_t len = (int64_t)start[e + 1] - s;
            if (s >= 0 && len >= 0 && s + len <= R) n = (int)len;
            else if (index == 0) atomicOr(status, kStatusBadIndex);
        }
        const int tiles = (n + height - 1) / height;
        int x = tiles;
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        const int at = index - before - (x - tiles);            // the tile's place in this lane's expert
        const uint32_t who = __ballot_sync(0xffffffffu, at >= 0 && at < tiles);
        if (who != 0) {
            const int src = __ffs(who) - 1;
            const int row = s + at * height, left = n - at * height;
            r.e = e0 + src;
            r.row = __shfl_sync(0xffffffffu, row, src);
            r.rows = __shfl_sync(0xffffffffu, left < height ? left : height, src);
            return r;
        }
        before += __shfl_sync(0xffffffffu, x, 31);
    }
    return r;
}

// Parameters of an input row and of a weight row.
struct RowParams { float as, ao, sx; int token; };              // token < 0: out of range
struct ColParams { float ws, wo, p3, bias; };                   // p3 = w_s S_w + K w_o

__device__ __forceinline__ RowParams row_params(const ExpertsArgs& g, int64_t row)
{
    RowParams p;
    const int64_t m = g.tokens != nullptr ? g.tokens[row] : row;
    p.token = m >= 0 && m < g.T ? (int)m : -1;
    p.as = p.ao = p.sx = __int_as_float(0x7fffffff);
    if (p.token >= 0) {
        const int64_t i = g.ep.n_aparam == 1 ? 0 : m;
        p.as = g.ep.a_scale[i]; p.ao = g.ep.a_offset[i]; p.sx = (float)g.a_sum[m];
    }
    return p;
}
__device__ __forceinline__ ColParams col_params(const ExpertsArgs& g, int64_t e, int64_t n)
{
    ColParams p;
    const int64_t at = e * g.N + n, i = g.ep.n_wparam == 1 ? 0 : at;
    p.ws = g.ep.w_scale[i]; p.wo = g.ep.w_offset[i];
    p.p3 = (float)((double)p.ws * (double)g.w_sum[at] + (double)g.K * (double)p.wo);
    p.bias = g.bias != nullptr ? g.bias[at] : 0.f;
    return p;
}

// y = w_s (a_s S) + (w_o (a_s S_x) + (p3 a_o + bias)): at most five roundings to a term, the same in both forms of the product.
__device__ __forceinline__ float affine(const RowParams& r, const ColParams& c, float S)
{
    return fmaf(c.ws, r.as * S, fmaf(c.wo, r.as * r.sx, fmaf(c.p3, r.ao, c.bias)));
}
// What the terms add up to in magnitude.
__device__ __forceinline__ float affine_size(const RowParams& r, const ColParams& c, float S)
{
    return fmaf(fabsf(c.ws), fabsf(r.as * S), fmaf(fabsf(c.wo), fabsf(r.as * r.sx), fmaf(fabsf(r.ao), fabsf(c.p3), fabsf(c.bias))));
}
// y / (1 + e^-y) by the approximate exponential and reciprocal (two and one units in the last place of 2^-23): within 6 units of 2^-24 |y|
// (the exponent's rounding, up to 2 |y| units of e^-y, comes with a factor e^-y / (1 + e^-y)^2).
__device__ __forceinline__ float fast_silu(float y)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(y * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return y * r;
}

__device__ __forceinline__ double exact_activation(double y, int act)
{
    switch (act) {
        case RTN_ACT_RELU: return y < 0.0 ? 0.0 : y;
        case RTN_ACT_GELU: return 0.5 * y * (1.0 + erf(y * 0.70710678118654752440));
        case RTN_ACT_GELU_TANH: return 0.5 * y * (1.0 + tanh(0.79788456080286535588 * (y + 0.044715 * y * y * y)));
        case RTN_ACT_SILU: return y / (1.0 + exp(-y));
        default: return y;
    }
}
__device__ __forceinline__ double exact_affine(const ExpertsArgs& g, int64_t m, int64_t e, int64_t n, float S)
{
    const int64_t at = e * g.N + n, i = g.ep.n_wparam == 1 ? 0 : at, j = g.ep.n_aparam == 1 ? 0 : m;
    const double ws = g.ep.w_scale[i], wo = g.ep.w_offset[i];
    return (double)g.ep.a_scale[j] * (ws * (double)S + wo * (double)g.a_sum[m]) + (double)g.ep.a_offset[j] * (ws * (double)g.w_sum[at] + (double)g.K * wo) +
           (g.bias != nullptr ? (double)g.bias[at] : 0.0);
}
// The value of output n of input row m in double, from its whole sums (S2: the second factor's).
static __device__ __noinline__ double exact_value(const ExpertsArgs& g, int64_t m, int64_t e, int64_t n, float S, float S2)
{
    const double v = exact_activation(exact_affine(g, m, e, n, S), g.act);
    return g.gated ? v * exact_affine(g, m, e, g.F + n, S2) : v;
}

constexpr float kUnit = 5.9604644775390625e-8f;                 // 2^-24

// One output, and (kCodes) the bits of its code.  The code is that of the exact value: a value nearer to a threshold than `err`, a bound on its
// own error (affine forms of five roundings, an activation of slope below 1.13 with 16 units of its own, the product), is worked out in
// double; of ordinary values a few in a million.
template <bool kCodes>
__device__ __forceinline__ float output_of(const ExpertsArgs& g, const RowParams& r, int64_t e, int64_t n, const ColParams& c, float S,
                                           const ColParams& c2, float S2, float lo, float hi, bool& up, bool& down)
{
    float a = affine(r, c, S), y2 = 1.f;
    const float y1 = a;
    if (g.act == RTN_ACT_SILU) a = fast_silu(a);
    else if (g.act != RTN_ACT_NONE) a = activation(a, g.act);
    float v = a;
    if (g.gated) { y2 = affine(r, c2, S2); v = a * y2; }
    if constexpr (kCodes) {
        float err = 6.f * affine_size(r, c, S) * 1.13f + 18.f * fabsf(y1);
        if (g.gated) err = fmaf(fabsf(y2), err, 6.f * fabsf(a) * affine_size(r, c2, S2) + fabsf(v));
        up = v > hi;
        down = !up && v < lo;
        const float d = fminf(fabsf(v - lo), fabsf(v - hi));
        if (!(d > 1.25f * kUnit * err)) {                       // (what overflowed or is NaN has such a bound)
            up = down = false;
            if (r.token >= 0) {
                const double x = exact_value(g, r.token, e, n, S, S2);
                up = x > (double)hi;
                down = !up && x < (double)lo;
            }
        }
    }
    return v;
}

#endif

}  // namespace rtn
