// Root-mean-square norms of the query and key heads and the rotation by position, one pass over both tensors:
//
//   y = x * w / sqrt(mean(x^2) + eps)            (w == NULL: y = x)
//   (y_a, y_b) <- (y_a c - y_b s, y_b c + y_a s)   for the R/2 pairs (a, b) of the head's first R elements,
//                                                  (c, s) = row positions[t] of the table
//
// with pairs (i, i + R/2) in the half layout and (2i, 2i + 1) in the interleaved one.
//
// Bound: DRAM, each element read and written once: 59 us at the size below are 5.7 TB/s, 0.88 of a plain copy's rate; small calls are
// bound by their launch (32 tokens: 2.4 us in a graph).  A group of lanes (a power of two, at most a warp) owns one head: a lane
// holds 16 bytes of it in registers, the sum of squares is a shuffle tree over the group, and in the half layout the
// lane reads its partner's 16 bytes as well (the line its own group just brought in: one load instead of a shuffle
// per element).  The cosines, sines and weights of a lane's elements are the same for every head of a token, so a group
// takes several heads of one token and reads them once.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"

namespace rtn {

namespace {

constexpr int kThreads = 64;
constexpr int kGenericWarps = 4;

__device__ __forceinline__ bool token_position(const RotaryArgs& g, int64_t t, int64_t& pos)
{
    pos = g.positions != nullptr ? g.positions[t] : t;
    return pos >= 0 && pos < g.table_rows;
}

// N consecutive floats, on a boundary of their own size (16 bytes at most).
template <int N>
__device__ __forceinline__ void load_floats(const float* p, float (&f)[N])
{
    if constexpr (N >= 4) {
        #pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(p + i));
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
    } else {
        const float2 v = __ldg(reinterpret_cast<const float2*>(p));
        f[0] = v.x; f[1] = v.y;
    }
}

__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src, bool real)       // zeros unless `real`
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// PG heads of one token per group of G lanes, HP at a time; CH 16-byte chunks per lane (head dimension up to 32 CH chunks).  Many
// heads are all asked for at once, into shared memory: it holds more of them in flight than registers do (16384 tokens of 32 + 8 heads
// of 128, bf16: 63 us instead of 74; with 18 CTAs per SM instead of 15, for a few spilled words of the weights, 59).
template <typename T, int CH, int HP, int PG, bool kHalf>
__global__ void __launch_bounds__(kThreads, PG > 2 && CH == 1 ? 18 : 1)
qk_norm_rotary_kernel(const RotaryArgs g, int G, int groups_q, int groups_k)
{
    constexpr bool kStage = PG > 2 && CH == 1;
    __shared__ uint4 stage[kStage ? PG : 1][kStage ? kThreads : 1];
    constexpr int V = Vec16<T>::N;
    const int lane_g = threadIdx.x & (G - 1);
    const unsigned item = blockIdx.x * (unsigned)(kThreads / G) + threadIdx.x / G;
    const unsigned per_token = groups_q + groups_k;
    const unsigned t = item / per_token;            // (32 bits hold it: the entry point bounds T (Hq + Hk))
    const bool live = t < g.T;                      // groups past the end stay for the warp's shuffles
    const int gi = (int)(item - t * per_token);
    const bool is_q = gi < groups_q;
    const int H = is_q ? g.Hq : g.Hk;
    const int h0 = (is_q ? gi : gi - groups_q) * PG;
    const int h1 = !live ? h0 : h0 + PG < H ? h0 + PG : H;
    const T* src = static_cast<const T*>(is_q ? g.q : g.k) + (int64_t)(live ? t : 0) * (is_q ? g.q_token : g.k_token);
    T* dst = static_cast<T*>(is_q ? g.out_q : g.out_k) + (int64_t)(live ? t : 0) * (is_q ? g.oq_token : g.ok_token);
    const int64_t s_head = is_q ? g.q_head : g.k_head, d_head = is_q ? g.oq_head : g.ok_head;
    const float* w = is_q ? g.q_weight : g.k_weight;
    const int nch = g.D / V, hch = g.R / 2 / V;     // chunks of a head, of half its rotated part

    // the first heads' elements (and, in the half layout, the partners'): everything below waits for them
    uint4 own[HP][CH], other[HP][kHalf ? CH : 1];
    const T* at = src + h0 * s_head + lane_g * V;
    T* to = dst + h0 * d_head + lane_g * V;
    auto load = [&](int h) {                        // heads h .. h + HP - 1, `at` on the first
        #pragma unroll
        for (int p = 0; p < HP; ++p)
            #pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int ch = lane_g + c * 32;
                own[p][c] = make_uint4(0, 0, 0, 0);
                if constexpr (kHalf) other[p][c] = make_uint4(0, 0, 0, 0);
                if (h + p < h1 && ch < nch) {
                    const uint4* row = reinterpret_cast<const uint4*>(at + p * s_head) + c * 32;
                    own[p][c] = *row;
                    if constexpr (kHalf) { if (ch < 2 * hch) other[p][c] = row[ch < hch ? hch : -hch]; }
                }
            }
    };
    if constexpr (kStage) {
        #pragma unroll
        for (int p = 0; p < PG; ++p) {
            const bool real = h0 + p < h1 && lane_g < nch;
            copy16_async((uint32_t)__cvta_generic_to_shared(&stage[p][threadIdx.x]), real ? at + p * s_head : src, real);
            if (p % HP == HP - 1) asm volatile("cp.async.commit_group;" ::: "memory");
        }
    } else load(h0);

    int64_t pos = 0;
    const bool pos_ok = !live || g.R == 0 || token_position(g, t, pos);
    if (!pos_ok && lane_g == 0) atomicOr(g.status, kStatusBadIndex);
    // y_e = (x_e A_e + o_e B_e) / rms with o the partner element: A = w cos, B = (partner's w) (-sin or sin), the same for every head
    float A[CH][V], B[CH][V];
    #pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int ch = lane_g + c * 32;
        const bool rot = ch < 2 * hch && pos_ok, second = ch >= hch;
        #pragma unroll
        for (int e = 0; e < V; ++e) {
            A[c][e] = pos_ok ? 1.f : __int_as_float(0x7fffffff);     // a position outside the table: NaN, never a wrong angle
            B[c][e] = 0.f;
        }
        if (rot) {
            const float* row = g.table + pos * g.R;
            if constexpr (kHalf) {
                const int f = (second ? ch - hch : ch) * V;
                load_floats<V>(row + f, A[c]);
                load_floats<V>(row + g.R / 2 + f, B[c]);
                #pragma unroll
                for (int e = 0; e < V; ++e) B[c][e] = second ? B[c][e] : -B[c][e];
            } else {
                float cs[V / 2], sn[V / 2];
                load_floats<V / 2>(row + ch * (V / 2), cs);
                load_floats<V / 2>(row + g.R / 2 + ch * (V / 2), sn);
                #pragma unroll
                for (int e = 0; e < V; ++e) { A[c][e] = cs[e / 2]; B[c][e] = (e & 1) ? sn[e / 2] : -sn[e / 2]; }
            }
        }
        if (w != nullptr && ch < nch) {
            float f[V];
            load_floats<V>(w + ch * V, f);
            #pragma unroll
            for (int e = 0; e < V; ++e) A[c][e] *= f[e];
            if (rot) {
                if constexpr (kHalf) load_floats<V>(w + (second ? ch - hch : ch + hch) * V, f);
                #pragma unroll
                for (int e = 0; e < V; ++e) B[c][e] *= kHalf ? f[e] : f[e ^ 1];
            }
        }
    }
    pair_t A2[CH][V / 2], B2[CH][V / 2];
    #pragma unroll
    for (int c = 0; c < CH; ++c)
        #pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            A2[c][e] = make_pair(A[c][2 * e], A[c][2 * e + 1]);
            B2[c][e] = make_pair(B[c][2 * e], B[c][2 * e + 1]);
        }
    const float inv_d = 1.f / (float)g.D;
    #pragma unroll (kStage ? PG / HP : 1)
    for (int done = 0; done < PG; done += HP) {     // (the same for every lane: they shuffle together)
        const int h = h0 + done;
        if constexpr (kStage) {
            // (the count of groups still on their way has to be a constant)
            if (done == 0) copies_wait<PG / HP - 1>();
            else if (done == HP) copies_wait<PG / HP - 2>();
            else if (done == 2 * HP) copies_wait<PG / HP - 3>();
            else copies_wait<0>();
            __syncwarp();
            #pragma unroll
            for (int p = 0; p < HP; ++p) {
                own[p][0] = stage[done + p][threadIdx.x];
                if constexpr (kHalf) {
                    other[p][0] = make_uint4(0, 0, 0, 0);
                    if (lane_g < 2 * hch) other[p][0] = stage[done + p][threadIdx.x + (lane_g < hch ? hch : -hch)];
                }
            }
        }
        pair_t y[HP][CH][V / 2];
        float r[HP];
        #pragma unroll
        for (int p = 0; p < HP; ++p) {
            pair_t ss = make_pair(0.f, 0.f);
            #pragma unroll
            for (int c = 0; c < CH; ++c) {
                pair_t x[V / 2], o[V / 2];
                Pairs16<T>::unpack(own[p][c], x);
                if constexpr (kHalf) {
                    Pairs16<T>::unpack(other[p][c], o);              // zero past the rotated part
                } else {
                    const bool rot = lane_g + c * 32 < 2 * hch;      // past it the neighbour's value stays out
                    #pragma unroll
                    for (int e = 0; e < V / 2; ++e) {
                        float a, b;
                        take_pair(x[e], a, b);
                        o[e] = make_pair(rot ? b : 0.f, rot ? a : 0.f);
                    }
                }
                #pragma unroll
                for (int e = 0; e < V / 2; ++e) {
                    ss = fma_pair(x[e], x[e], ss);
                    y[p][c][e] = fma_pair(x[e], A2[c][e], mul_pair(o[e], B2[c][e]));
                }
            }
            float a, b;
            take_pair(ss, a, b);
            r[p] = a + b;
        }
        at += HP * s_head;
        if constexpr (!kStage) {
            if (done + HP < PG) load(h + HP);
            __syncwarp();                           // in place, a lane's elements are read by its partner before it writes them
        }
        if (w != nullptr) {
            #pragma unroll
            for (int d = 16; d > 0; d >>= 1)
                if (d < G) {
                    #pragma unroll
                    for (int p = 0; p < HP; ++p) r[p] += __shfl_xor_sync(0xffffffffu, r[p], d);
                }
        }
        #pragma unroll
        for (int p = 0; p < HP; ++p) {
            const float s = w != nullptr ? rsqrtf(fmaf(r[p], inv_d, g.eps)) : 1.f;
            #pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (h + p >= h1 || lane_g + c * 32 >= nch) continue;
                #pragma unroll
                for (int e = 0; e < V / 2; ++e) y[p][c][e] = mul_pair(y[p][c][e], make_pair(s, s));
                reinterpret_cast<uint4*>(to + p * d_head)[c * 32] = Pairs16<T>::pack(y[p][c]);
            }
        }
        to += HP * d_head;
    }
}

// Any head dimension, stride and alignment: a warp per (token, head), the head staged in shared memory as fp32.
template <typename T>
__global__ void __launch_bounds__(kGenericWarps * 32)
qk_norm_rotary_generic_kernel(const RotaryArgs g)
{
    __shared__ float stage[kGenericWarps][kRotaryMaxDim];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* x = stage[warp];
    const int heads = g.Hq + g.Hk, half = g.R / 2;
    const int64_t item = (int64_t)blockIdx.x * kGenericWarps + warp;
    if (item >= g.T * heads) return;
    const int64_t t = item / heads;
    int h = (int)(item - t * heads);
    const bool is_q = h < g.Hq;
    if (!is_q) h -= g.Hq;
    const T* src = static_cast<const T*>(is_q ? g.q : g.k) + t * (is_q ? g.q_token : g.k_token) + h * (is_q ? g.q_head : g.k_head);
    T* dst = static_cast<T*>(is_q ? g.out_q : g.out_k) + t * (is_q ? g.oq_token : g.ok_token) + h * (is_q ? g.oq_head : g.ok_head);
    const float* w = is_q ? g.q_weight : g.k_weight;
    float ss = 0.f;
    for (int e = lane; e < g.D; e += 32) {
        const float v = to_f32(src[e]);
        x[e] = v;
        ss = fmaf(v, v, ss);
    }
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);      // also orders the stores to x before the reads
    __syncwarp();
    int64_t pos = 0;
    const bool pos_ok = g.R == 0 || token_position(g, t, pos);
    if (!pos_ok && lane == 0) atomicOr(g.status, kStatusBadIndex);
    float r = w != nullptr ? rsqrtf(ss / (float)g.D + g.eps) : 1.f;
    if (!pos_ok) r = __int_as_float(0x7fffffff);
    const float* row = g.table + (pos_ok ? pos : 0) * g.R;
    for (int e = lane; e < g.D; e += 32) {
        float y = x[e] * (w != nullptr ? w[e] : 1.f);
        if (e < g.R && pos_ok) {
            const bool is_half = g.layout == RTN_ROTARY_HALF;
            const int f = is_half ? (e < half ? e : e - half) : e >> 1;
            const bool second = is_half ? e >= half : (e & 1);
            const int pe = is_half ? (second ? e - half : e + half) : e ^ 1;
            const float o = x[pe] * (w != nullptr ? w[pe] : 1.f);
            const float s = row[half + f];
            y = fmaf(y, row[f], second ? o * s : -o * s);
        }
        dst[e] = from_f32<T>(y * r);
    }
}

// Row p of the table: cos(p f_i) and sin(p f_i), i < R/2, times the amplitude; angles in double (p f_i passes 2^24).
//   f_i = base^(-2i/R);  LINEAR: f_i / factor;  BASE: base * factor^(R/(R-2)) in place of base;
//   PARTS: by the turns f_i makes over the original context, f_i above `high`, f_i / factor below `low`, a ramp between
__global__ void rotary_table_kernel(float* __restrict__ table, int64_t rows, int R, double base, int kind, double factor,
                                    double original, double low, double high, double amplitude)
{
    const int half = R / 2;
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= rows * half) return;
    const int64_t p = i / half;
    const int j = (int)(i - p * half);
    if (kind == RTN_ROTARY_SCALE_BASE) base *= pow(factor, (double)R / (double)(R - 2));
    double f = exp2(-2.0 * (double)j / (double)R * log2(base));
    if (kind == RTN_ROTARY_SCALE_LINEAR) f /= factor;
    if (kind == RTN_ROTARY_SCALE_PARTS) {
        const double turns = original * f / 6.283185307179586476925;
        double keep = (turns - low) / (high - low);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        f = f * (keep + (1.0 - keep) / factor);
    }
    double s, c;
    sincos((double)p * f, &s, &c);
    table[p * R + j] = (float)(amplitude * c);
    table[p * R + half + j] = (float)(amplitude * s);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename T, int CH, int HP, int PG>
cudaError_t launch_vec(const RotaryArgs& g, int G, cudaStream_t s)
{
    const int gq = (g.Hq + PG - 1) / PG, gk = (g.Hk + PG - 1) / PG;
    const int64_t items = g.T * (gq + gk), per_cta = kThreads / G;
    const unsigned grid = (unsigned)((items + per_cta - 1) / per_cta);
    if (g.layout == RTN_ROTARY_HALF) qk_norm_rotary_kernel<T, CH, HP, PG, true><<<grid, kThreads, 0, s>>>(g, G, gq, gk);
    else qk_norm_rotary_kernel<T, CH, HP, PG, false><<<grid, kThreads, 0, s>>>(g, G, gq, gk);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_typed(const RotaryArgs& g, cudaStream_t s)
{
    constexpr int V = Vec16<T>::N;
    // 16-byte path: whole chunks in the head and in each half of its rotated part, every row on a 16-byte boundary
    const int64_t strides = g.q_token | g.q_head | g.k_token | g.k_head | g.oq_token | g.oq_head | g.ok_token | g.ok_head;
    const bool vec = g.D % V == 0 && (g.R / 2) % V == 0 && strides % V == 0 && g.D / V <= 64 && aligned16(g.q) &&
                     aligned16(g.k) && aligned16(g.out_q) && aligned16(g.out_k) && aligned16(g.table) &&
                     aligned16(g.q_weight) && aligned16(g.k_weight);
    if (!vec) {
        const int64_t items = g.T * (g.Hq + g.Hk);
        qk_norm_rotary_generic_kernel<T><<<(unsigned)((items + kGenericWarps - 1) / kGenericWarps), kGenericWarps * 32, 0, s>>>(g);
        return cudaGetLastError();
    }
    const int nch = g.D / V;
    int G = 1;
    while (G < nch && G < 32) G *= 2;
    // Few tokens: a head per group, for the most groups; many: eight, for the fewest table and weight reads.
    const int64_t warps = g.T * (g.Hq + g.Hk) * G / 32;
    const int per_group = warps > (int64_t)device_sm_count() * 128 ? 8 : warps > (int64_t)device_sm_count() * 32 ? 2 : 1;
    if (nch > 32) return per_group == 1 ? launch_vec<T, 2, 1, 1>(g, G, s) : launch_vec<T, 2, 1, 8>(g, G, s);
    return per_group == 1 ? launch_vec<T, 1, 1, 1>(g, G, s) : per_group == 2 ? launch_vec<T, 1, 2, 2>(g, G, s) : launch_vec<T, 1, 2, 8>(g, G, s);
}

}  // namespace

cudaError_t launch_qk_norm_rotary(const RotaryArgs& g, cudaStream_t s)
{
    return with_dtype(g.dtype, [&](auto t) { return launch_typed<decltype(t)>(g, s); });
}

cudaError_t launch_rotary_table(float* table, int64_t rows, int R, double base, int kind, double factor, double original,
                                double low, double high, double amplitude, cudaStream_t s)
{
    const int64_t n = rows * (R / 2);
    rotary_table_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(table, rows, R, base, kind, factor, original, low, high, amplitude);
    return cudaGetLastError();
}

}  // namespace rtn
