// The norms after one block and before the next, with the block's gate, its residual and the experts' weighted sum, and the codes of the
// result: a CTA per token, the token's values in registers between the passes.
//
// Bound: HBM, every input and output once.
//
// Codes are those of the exact value.  Beside each value runs a bound on its rounding error in units of u = 2^-24 (to first order):
//   y = sum_j w_j x_j, one rounding per term           E_y <= k sum_j |w_j x_j|   (0 without weights)
//   1/sqrt(mean + eps) of a sum of squares over a tree  relative: (half of the tree's depth) + |E| / |.| (of the vector norms)
// and so on through gate, scale and residual.  A value nearer to a threshold than its bound, or one that is not finite, makes the CTA work
// the token's codes out again in double; of tokens of 2048 normal values about one in a hundred.
#include "rtn_internal.cuh"
#include "rtn_epilogue.cuh"

namespace rtn {

namespace {

constexpr float kUnit = 5.9604644775390625e-8f;                // 2^-24
constexpr int kMaxWarps = 32;

// EV adjacent elements as fp32: 16-byte loads where EV > 1 (the launcher saw to the alignment).
template <typename T, int EV>
__device__ __forceinline__ void load_values(const void* base, int64_t at, float (&f)[EV])
{
    const T* p = static_cast<const T*>(base) + at;
    if constexpr (EV == 1) f[0] = to_f32(*p);
    else {
        constexpr int N = Vec16<T>::N;
        static_assert(EV % N == 0, "whole vectors");
        #pragma unroll
        for (int i = 0; i < EV / N; ++i) {
            float part[N];
            Vec16<T>::unpack(reinterpret_cast<const uint4*>(p)[i], part);
            #pragma unroll
            for (int j = 0; j < N; ++j) f[i * N + j] = part[j];
        }
    }
}
template <typename T, int EV>
__device__ __forceinline__ void store_values(void* base, int64_t at, const float (&f)[EV])
{
    T* p = static_cast<T*>(base) + at;
    if constexpr (EV == 1) *p = from_f32<T>(f[0]);
    else {
        constexpr int N = Vec16<T>::N;
        #pragma unroll
        for (int i = 0; i < EV / N; ++i) {
            float part[N];
            #pragma unroll
            for (int j = 0; j < N; ++j) part[j] = f[i * N + j];
            reinterpret_cast<uint4*>(p)[i] = Vec16<T>::pack(part);
        }
    }
}
template <int EV>
__device__ __forceinline__ void load_params(const float* p, int at, float (&f)[EV])     // (of W values, 4-byte aligned)
{
    #pragma unroll
    for (int i = 0; i < EV; ++i) f[i] = p[at + i];
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

__device__ __forceinline__ float gate_of(float z, int kind)
{
    if (kind == RTN_GATE_LINEAR) return z;
    const float s = 1.f / (1.f + expf(-z));
    return kind == RTN_GATE_SIGMOID ? s : z * s;
}

// Roundings of a sum of squares: per thread, two shuffle trees, and the mean, root and quotient after it.
template <int NV, int EV> constexpr float kRootUnits = 0.5f * (NV * EV + 10) + 5.f;

// h and n of token t.  slack receives the bound on n's error, where kTrack asks for it.
template <typename TB, typename TS, int EV, int NV, bool kTrack>
__device__ __forceinline__ void norm_row(const NormArgs& g, int64_t t, float* red, float (&h)[NV][EV], float (&n)[NV][EV], float (&slack)[NV][EV])
{
    const int W = g.W, step = blockDim.x * EV, first = threadIdx.x * EV;
    const float k_units = g.place != nullptr ? (float)g.k : 0.f;
    float zero = 0.f, ss = 0.f, sm = 0.f;
    #pragma unroll
    for (int v = 0; v < NV; ++v)
        #pragma unroll
        for (int i = 0; i < EV; ++i) h[v][i] = slack[v][i] = 0.f;
    // y in h, the sum of its terms' magnitudes in slack
    if (g.branch != nullptr) {
        #pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = first + v * step;
            if (c >= W) continue;
            if (g.place == nullptr) {
                load_values<TB, EV>(g.branch, t * g.branch_stride + c, h[v]);
            } else {
                #pragma unroll 4
                for (int j = 0; j < g.k; ++j) {
                    const int64_t row = g.place[t * g.k + j];
                    float w = g.weights != nullptr ? g.weights[t * g.k + j] : 1.f;
                    if (row < 0) continue;
                    float x[EV];
                    if (row < g.R) load_values<TB, EV>(g.branch, row * g.branch_stride + c, x);
                    else {
                        w = __int_as_float(0x7fffffff);
                        #pragma unroll
                        for (int i = 0; i < EV; ++i) x[i] = w;
                    }
                    #pragma unroll
                    for (int i = 0; i < EV; ++i) {
                        h[v][i] = fmaf(w, x[i], h[v][i]);
                        if constexpr (kTrack) slack[v][i] = fmaf(fabsf(w), fabsf(x[i]), slack[v][i]);
                    }
                }
            }
        }
    }
    float post = 1.f, post_units = 0.f;
    if (g.post_weight != nullptr) {
        #pragma unroll
        for (int v = 0; v < NV; ++v)
            #pragma unroll
            for (int i = 0; i < EV; ++i) {
                ss = fmaf(h[v][i], h[v][i], ss);
                if constexpr (kTrack) sm = fmaf(slack[v][i], slack[v][i], sm);
            }
        block_sums(ss, kTrack ? sm : zero, red);
        post = 1.f / sqrtf(ss / (float)W + g.eps);
        if constexpr (kTrack) post_units = kRootUnits<NV, EV> + 2.f + (ss > 0.f ? k_units * sqrtf(sm / ss) : 0.f);
    }
    ss = sm = 0.f;
    #pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = first + v * step;
        if (c >= W) continue;
        float f[EV];
        #pragma unroll
        for (int i = 0; i < EV; ++i) f[i] = 1.f;
        float units = 0.f;                                      // roundings of the factor and its product
        if (g.branch != nullptr) {
            float p[EV];
            if (g.post_weight != nullptr) {
                load_params<EV>(g.post_weight, c, p);
                #pragma unroll
                for (int i = 0; i < EV; ++i) f[i] = post * p[i];
                units = 2.f;
            }
            if (g.gate != nullptr) {
                load_values<TB, EV>(g.gate, t * g.gate_stride + c, p);
                #pragma unroll
                for (int i = 0; i < EV; ++i) f[i] *= gate_of(p[i], g.gate_kind);
                units += 12.f;
            }
            if (g.scale != nullptr) {
                if (g.n_scale == 1) {
                    #pragma unroll
                    for (int i = 0; i < EV; ++i) f[i] *= g.scale[0];
                } else {
                    load_params<EV>(g.scale, c, p);
                    #pragma unroll
                    for (int i = 0; i < EV; ++i) f[i] *= p[i];
                }
                units += 1.f;
            }
        }
        float r[EV];
        #pragma unroll
        for (int i = 0; i < EV; ++i) r[i] = 0.f;
        if (g.residual != nullptr) load_values<TS, EV>(g.residual, t * g.residual_stride + c, r);
        #pragma unroll
        for (int i = 0; i < EV; ++i) {
            const float y = h[v][i];
            h[v][i] = fmaf(f[i], y, r[i]);
            if constexpr (kTrack) {
                slack[v][i] = fmaf(fabsf(f[i]), fmaf(k_units, slack[v][i], (post_units + units) * fabsf(y)), fabsf(h[v][i]));
                sm = fmaf(slack[v][i], slack[v][i], sm);
            }
            ss = fmaf(h[v][i], h[v][i], ss);
        }
    }
    float pre = 1.f, pre_units = 0.f;
    if (g.norm_weight != nullptr) {
        block_sums(ss, kTrack ? sm : zero, red);
        pre = 1.f / sqrtf(ss / (float)W + g.eps);
        if constexpr (kTrack) pre_units = kRootUnits<NV, EV> + 4.f + (ss > 0.f ? sqrtf(sm / ss) : 0.f);
    }
    #pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = first + v * step;
        #pragma unroll
        for (int i = 0; i < EV; ++i) n[v][i] = h[v][i];
        if (c >= W || g.norm_weight == nullptr) continue;
        float p[EV];
        load_params<EV>(g.norm_weight, c, p);
        #pragma unroll
        for (int i = 0; i < EV; ++i) {
            const float f = pre * p[i];
            n[v][i] = f * h[v][i];
            if constexpr (kTrack) slack[v][i] = fmaf(fabsf(f), slack[v][i], pre_units * fabsf(n[v][i]));
        }
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
            near |= !(d > 1.25f * kUnit * slack[v][i]) || !(fabsf(x) < 1e37f);
        }
    }
    return near;
}

// The codes of one token in double, whatever the types: the inputs are read again in each pass.
__device__ __forceinline__ double exact_y(const NormArgs& g, int64_t t, int c)
{
    if (g.branch == nullptr) return 0.0;
    if (g.place == nullptr) return (double)load_as_f32(g.branch, t * g.branch_stride + c, g.dtype);
    double y = 0.0;
    for (int j = 0; j < g.k; ++j) {
        const int64_t row = g.place[t * g.k + j];
        if (row < 0) continue;
        if (row >= g.R) return __longlong_as_double(0x7fffffffffffffffll);
        y = fma(g.weights != nullptr ? (double)g.weights[t * g.k + j] : 1.0, (double)load_as_f32(g.branch, row * g.branch_stride + c, g.dtype), y);
    }
    return y;
}
__device__ __forceinline__ double exact_h(const NormArgs& g, int64_t t, int c, double post)
{
    double y = exact_y(g, t, c);
    if (g.post_weight != nullptr) y *= post * (double)g.post_weight[c];
    if (g.gate != nullptr) {
        const double z = (double)load_as_f32(g.gate, t * g.gate_stride + c, g.dtype), s = 1.0 / (1.0 + exp(-z));
        y *= g.gate_kind == RTN_GATE_LINEAR ? z : g.gate_kind == RTN_GATE_SIGMOID ? s : z * s;
    }
    if (g.scale != nullptr) y *= (double)g.scale[g.n_scale == 1 ? 0 : c];
    return g.residual != nullptr ? (double)load_as_f32(g.residual, t * g.residual_stride + c, g.stream_dtype) + y : y;
}
static __device__ __noinline__ int exact_codes(const NormArgs& g, int64_t t, double* red, uint8_t* row)
{
    double post = 1.0, pre = 1.0, none = 0.0;
    if (g.post_weight != nullptr) {
        double ss = 0.0;
        for (int c = threadIdx.x; c < g.W; c += blockDim.x) { const double y = exact_y(g, t, c); ss = fma(y, y, ss); }
        block_sums(ss, none, red);
        post = 1.0 / sqrt(ss / (double)g.W + (double)g.eps);
    }
    if (g.norm_weight != nullptr) {
        double ss = 0.0;
        for (int c = threadIdx.x; c < g.W; c += blockDim.x) { const double h = exact_h(g, t, c, post); ss = fma(h, h, ss); }
        none = 0.0;
        block_sums(ss, none, red);
        pre = 1.0 / sqrt(ss / (double)g.W + (double)g.eps);
    }
    int sum = 0;
    const int width = (g.W + kBlockCodes - 1) / kBlockCodes * kBlockCodes;
    for (int c0 = threadIdx.x & ~31; c0 < width; c0 += blockDim.x) {
        const int c = c0 + (threadIdx.x & 31);
        bool up = false, down = false;
        if (c < g.W) {
            double n = exact_h(g, t, c, post);
            if (g.norm_weight != nullptr) n *= pre * (double)g.norm_weight[c];
            const int i = g.n_thr == 1 ? 0 : c;
            up = n > (double)g.t_hi[i];
            down = !up && n < (double)g.t_lo[i];
        }
        const uint32_t a = __ballot_sync(0xffffffffu, up), b = __ballot_sync(0xffffffffu, down);
        if ((threadIdx.x & 31) == 0) {
            uint32_t* at = reinterpret_cast<uint32_t*>(row + c0 / kBlockCodes * kBlockBytes + c0 % kBlockCodes / 8);
            at[0] = a | b;
            at[4] = a;
            sum += __popc(a) - __popc(b);
        }
    }
    return sum;
}

template <typename TB, typename TS, int EV, int NV, bool kCodes>
__global__ void __launch_bounds__(1024)
block_norm_kernel(const __grid_constant__ NormArgs g)
{
    __shared__ double red[2 * kMaxWarps];
    const int64_t t = blockIdx.x;
    float h[NV][EV], n[NV][EV], slack[NV][EV];
    norm_row<TB, TS, EV, NV, kCodes>(g, t, reinterpret_cast<float*>(red), h, n, slack);
    if constexpr (kCodes) {
        uint32_t up, down;
        const bool near = code_row<EV, NV>(g, n, slack, up, down);
        const int blocks = (g.W + kBlockCodes - 1) / kBlockCodes;
        uint8_t* row = g.out_packed + t * blocks * kBlockBytes;
        int own = __popc(up) - __popc(down);
        if (__syncthreads_or(near)) {
            own = exact_codes(g, t, red, row);
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
                    const uint32_t a = __ballot_sync(0xffffffffu, up >> v & 1), b = __ballot_sync(0xffffffffu, down >> v & 1);
                    if ((threadIdx.x & 31) == 0 && c < blocks * kBlockCodes) {
                        uint32_t* at = reinterpret_cast<uint32_t*>(row + c / kBlockCodes * kBlockBytes + c % kBlockCodes / 8);
                        at[0] = a | b;
                        at[4] = a;
                    }
                }
            }
        }
        float sum = (float)own, none = 0.f;                     // (whole numbers below 2^24)
        block_sums(sum, none, reinterpret_cast<float*>(red));
        if (threadIdx.x == 0) g.out_sum[t] = (int)sum;
    }
    #pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = threadIdx.x * EV + v * blockDim.x * EV;
        if (c >= g.W) continue;
        if (g.stream_out != nullptr) store_values<TS, EV>(g.stream_out, t * g.stream_stride + c, h[v]);
        if (g.normed != nullptr) store_values<TB, EV>(g.normed, t * g.normed_stride + c, n[v]);
    }
    if (threadIdx.x == 0 && g.place != nullptr) {
        bool bad = false;
        for (int j = 0; j < g.k; ++j) bad |= g.place[t * g.k + j] >= g.R;
        if (bad) atomicOr(g.status, kStatusBadIndex);
    }
}

template <typename TB, typename TS, int EV, int NV>
cudaError_t launch_values(const NormArgs& g, cudaStream_t s)
{
    const int width = (g.W + kBlockCodes - 1) / kBlockCodes * kBlockCodes;         // (the padding of a packed row is written too)
    const int threads = ((width + EV * NV - 1) / (EV * NV) + 31) / 32 * 32;
    if (g.out_packed != nullptr) block_norm_kernel<TB, TS, EV, NV, true><<<(unsigned)g.T, threads, 0, s>>>(g);
    else block_norm_kernel<TB, TS, EV, NV, false><<<(unsigned)g.T, threads, 0, s>>>(g);
    return cudaGetLastError();
}

template <typename TB, typename TS>
cudaError_t launch_types(const NormArgs& g, cudaStream_t s)
{
    auto vec = [](const void* p, int64_t stride, size_t e) {
        return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride * (int64_t)e % 16 == 0);
    };
    const bool wide = g.W % 8 == 0 && vec(g.branch, g.branch_stride, sizeof(TB)) && vec(g.gate, g.gate_stride, sizeof(TB)) &&
                      vec(g.normed, g.normed_stride, sizeof(TB)) && vec(g.residual, g.residual_stride, sizeof(TS)) &&
                      vec(g.stream_out, g.stream_stride, sizeof(TS));
    if (wide) return g.W <= 8192 ? launch_values<TB, TS, 8, 1>(g, s) : launch_values<TB, TS, 8, 2>(g, s);
    if (g.W <= 4096) return launch_values<TB, TS, 1, 4>(g, s);
    return launch_values<TB, TS, 1, 16>(g, s);
}

}  // namespace

cudaError_t launch_block_norm(const NormArgs& g, cudaStream_t s)
{
    return with_dtype(g.dtype, [&](auto b) {
        return with_dtype(g.stream_dtype, [&](auto t) { return launch_types<decltype(b), decltype(t)>(g, s); });
    });
}

}  // namespace rtn
