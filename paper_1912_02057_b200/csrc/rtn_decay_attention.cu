// Linear attention with a decay l = exp(log_decay[h]) for each head h, per sequence and query head:
//
//   S_t = l S_{t-1} + k_t v_t^T        (S: Dk x Dv, fp32)
//   o_t = scale q_t^T S_t
//
// decay_step_kernel: one token per sequence.  Bound: DRAM, the fp32 state read and written once (8 Dk Dv bytes per head
//   against 4 Dk Dv operations).
// decay_recurrent_kernel: whole prompts token by token with the state in registers; any type, head dimension and
//   stride.  Bound: the FMA pipe (two FMAs per state element and token).
#include "rtn_internal.cuh"
#include "rtn_types.cuh"
#include "rtn_decay.cuh"

namespace rtn {

namespace {

// ------------------------------------------------------------------------------------------------ single tokens

constexpr int kStepThreads = 256;
constexpr int kStepBatch = 8;           // state vectors a thread has in flight

// CTA = (sequence, head, slice of VW-element column groups).  Thread (r, c) owns columns VW c .. of the rows r, r + nr, ...:
// a warp reads whole sectors of consecutive rows, and every state element is touched once.
template <typename T, int VW>
__global__ void __launch_bounds__(kStepThreads)
decay_step_kernel(const DecayArgs g, int slice, int slices)
{
    __shared__ float sq[kDecayMaxDim], sk[kDecayMaxDim], red[kStepThreads * VW];
    int64_t bid = blockIdx.x;
    const int sl = (int)(bid % slices); bid /= slices;
    const int h = (int)(bid % g.H);
    const int64_t b = bid / g.H;
    const int hk = h / (g.H / g.Hk);
    const int64_t slot = g.slot != nullptr ? g.slot[b] : b;
    const int c0 = sl * slice, cols = g.Dv - c0 < slice ? g.Dv - c0 : slice;
    T* out = static_cast<T*>(g.out) + b * g.o_token + h * g.o_head + c0;
    if (slot < 0 || slot >= g.n_slots) {
        for (int c = threadIdx.x; c < cols; c += kStepThreads) out[c] = from_f32<T>(slot < 0 ? 0.f : __int_as_float(0x7fffffff));
        if (slot >= g.n_slots && threadIdx.x == 0) atomicOr(g.status, kStatusBadIndex);
        return;
    }
    const T* q = static_cast<const T*>(g.q) + b * g.q_token + h * g.q_head;
    const T* k = static_cast<const T*>(g.k) + b * g.k_token + hk * g.k_head;
    const T* v = static_cast<const T*>(g.v) + b * g.v_token + hk * g.v_head + c0;
    const int cw = (cols + VW - 1) / VW, nr = kStepThreads / cw;
    const int c = threadIdx.x % cw, r0 = threadIdx.x / cw;
    const int64_t base = (slot * g.H + h) * (int64_t)g.Dk * g.Dv + c0 + c * VW;
    const bool mine = r0 < nr;
    for (int i = threadIdx.x; i < g.Dk; i += kStepThreads) { sq[i] = to_f32(q[i]); sk[i] = to_f32(k[i]); }
    float vv[VW], acc[VW];
    #pragma unroll
    for (int e = 0; e < VW; ++e) { vv[e] = mine ? to_f32(v[c * VW + e]) : 0.f; acc[e] = 0.f; }
    const float l = expf(g.log_decay[h]);
    __syncthreads();
    for (int r = r0; mine && r < g.Dk; r += kStepBatch * nr) {
        float s[kStepBatch][VW];
        #pragma unroll
        for (int i = 0; i < kStepBatch; ++i) {
            const int row = r + i * nr;
            #pragma unroll
            for (int e = 0; e < VW; ++e) s[i][e] = 0.f;
            if (g.state != nullptr && row < g.Dk) {
                const float* p = g.state + base + (int64_t)row * g.Dv;
                if constexpr (VW == 4) {
                    const float4 f = *reinterpret_cast<const float4*>(p);
                    s[i][0] = f.x; s[i][1] = f.y; s[i][2] = f.z; s[i][3] = f.w;
                } else s[i][0] = *p;
            }
        }
        #pragma unroll
        for (int i = 0; i < kStepBatch; ++i) {
            const int row = r + i * nr;
            if (row >= g.Dk) continue;
            const float kk = sk[row], qq = sq[row];
            #pragma unroll
            for (int e = 0; e < VW; ++e) {
                s[i][e] = g.state != nullptr ? fmaf(l, s[i][e], kk * vv[e]) : kk * vv[e];
                acc[e] = fmaf(qq, s[i][e], acc[e]);
            }
            float* p = g.state_out + base + (int64_t)row * g.Dv;
            if constexpr (VW == 4) *reinterpret_cast<float4*>(p) = make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
            else *p = s[i][0];
        }
    }
    #pragma unroll
    for (int e = 0; e < VW; ++e) red[threadIdx.x * VW + e] = acc[e];
    __syncthreads();
    for (int j = threadIdx.x; j < cols; j += kStepThreads) {
        float o = 0.f;
        for (int r = 0; r < nr; ++r) o += red[(r * cw) * VW + j];
        out[j] = from_f32<T>(g.scale * o);
    }
}

template <typename T>
cudaError_t launch_step_typed(const DecayArgs& g, cudaStream_t s)
{
    const bool vec = g.Dv % 4 == 0 && (reinterpret_cast<uintptr_t>(g.state) & 15) == 0 && (reinterpret_cast<uintptr_t>(g.state_out) & 15) == 0;
    // few heads in all: 32 columns (whole 128-byte rows) per CTA, so that more SMs pull on the memory
    const int slice = g.B * g.H < 2 * device_sm_count() ? 32 : kDecayMaxDim;
    const int slices = (g.Dv + slice - 1) / slice;
    const unsigned grid = (unsigned)(g.B * g.H * slices);
    if (vec) decay_step_kernel<T, 4><<<grid, kStepThreads, 0, s>>>(g, slice, slices);
    else decay_step_kernel<T, 1><<<grid, kStepThreads, 0, s>>>(g, slice, slices);
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------------------------ prompts, token by token

constexpr int kRecWarps = 4;            // each holds a quarter of the state's rows
constexpr int kRecThreads = kRecWarps * 32;
constexpr int kRecTile = 8;             // tokens staged at a time, at most (16: 8 x 2048 tokens of 32 heads 1500 us instead of 1160)

struct RecPlan {
    int64_t seg_len;        // tokens of a segment
    int segments;           // of the longest sequence
    float* local;           // [B][H][segments][Dk][Dv]: the state before the first segment, then what each but the last adds to it
};

// l^n from log2 l; n = 0 gives 1 for every l.
__device__ __forceinline__ float power(float g2, float n) { return n == 0.f ? 1.f : exp2f(n * g2); }

// Column(s) of the state in the lanes of four warps, rows in registers by pairs.  Within a tile of tokens i = 0, 1, ... the state is kept
// relative to the tile's first token,
//   S_i = l^i S'_i,   S'_i = S'_(i-1) + (l^-i k_i) v_i^T,   o_i = (l^i q_i)^T S'_i,
// which leaves one FMA per element for the update and one for the output, two elements to an instruction.  A tile ends before
// l^-i passes e^60; at l = 0 it is one token.
template <typename T, int ROWS, int COLS, bool kStates>
__global__ void __launch_bounds__(kRecThreads)
decay_recurrent_kernel(const DecayArgs g, const RecPlan p)
{
    constexpr int DK = ROWS * kRecWarps, DV = COLS * 32;
    __shared__ __align__(16) float sq[kStates ? 1 : kRecTile][DK], sk[kRecTile][DK];
    __shared__ float sv[kRecTile][DV], so[kStates ? 1 : kRecTile][kRecWarps][DV], grow[kRecTile], shrink[kRecTile];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int h = blockIdx.y, hk = h / (g.H / g.Hk);
    const int slices = (g.Dv + DV - 1) / DV;
    const int c0 = (int)(blockIdx.z % slices) * DV, seg = (int)(blockIdx.z / slices);
    const int64_t b = blockIdx.x;
    int64_t first, len, slot;
    if (!sequence_bounds(g, b, first, len, slot)) {
        if (!kStates && threadIdx.x == 0 && seg == 0) atomicOr(g.status, kStatusBadIndex);
        return;
    }
    const int64_t s0 = (int64_t)seg * p.seg_len;
    if (seg > 0 && s0 >= len) return;
    const bool last_seg = s0 + p.seg_len >= len;
    if (kStates && (last_seg || slot < 0)) return;
    const int64_t n_tok = last_seg ? len - s0 : p.seg_len;
    first += s0;
    const int cols = g.Dv - c0 < DV ? g.Dv - c0 : DV;
    T* out = static_cast<T*>(g.out) + first * g.o_token + h * g.o_head + c0;
    if (slot < 0) {
        for (int64_t i = threadIdx.x; i < n_tok * cols; i += kRecThreads) out[(i / cols) * g.o_token + i % cols] = from_f32<T>(0.f);
        return;
    }
    const T* q = static_cast<const T*>(g.q) + first * g.q_token + h * g.q_head;
    const T* k = static_cast<const T*>(g.k) + first * g.k_token + hk * g.k_head;
    const T* v = static_cast<const T*>(g.v) + first * g.v_token + hk * g.v_head + c0;
    const float g2 = g.log_decay[h] * 1.4426950408889634f;
    const float reach = 86.f / fmaxf(fabsf(g2), 1e-6f);                     // steps until |log2| passes 86 (about e^60)
    const int tile = reach >= (float)(kRecTile - 1) ? kRecTile : 1 + (int)reach;
    const int64_t base = (slot * g.H + h) * (int64_t)g.Dk * g.Dv + c0 + lane;
    const int64_t slice = (int64_t)g.Dk * g.Dv, local_base = (b * g.H + h) * (int64_t)p.segments * slice + c0 + lane;
    pair_t S[COLS][ROWS / 2];
    auto store = [&](float* dst) {
        #pragma unroll
        for (int i = 0; i < ROWS; i += 2)
            #pragma unroll
            for (int c = 0; c < COLS; ++c) {
                float s[2];
                take_pair(S[c][i / 2], s[0], s[1]);
                #pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = warp * ROWS + i + e;
                    if (r < g.Dk && lane + 32 * c < cols) dst[(int64_t)r * g.Dv + 32 * c] = s[e];
                }
            }
    };
    {
        // the given state and what the segments before this one added, one whole slice after the other (every load of a slice in flight)
        #pragma unroll
        for (int c = 0; c < COLS; ++c)
            #pragma unroll
            for (int i = 0; i < ROWS / 2; ++i) S[c][i] = make_pair(0.f, 0.f);
        auto add = [&](const float* src, float w) {
            float x[COLS][ROWS];
            #pragma unroll
            for (int c = 0; c < COLS; ++c)
                #pragma unroll
                for (int i = 0; i < ROWS; ++i)
                    x[c][i] = warp * ROWS + i < g.Dk && lane + 32 * c < cols ? src[(int64_t)(warp * ROWS + i) * g.Dv + 32 * c] : 0.f;
            #pragma unroll
            for (int c = 0; c < COLS; ++c)
                #pragma unroll
                for (int i = 0; i < ROWS; i += 2) S[c][i / 2] = fma_pair(make_pair(w, w), make_pair(x[c][i], x[c][i + 1]), S[c][i / 2]);
        };
        if constexpr (kStates) {
            // The last segment's CTA writes state_out, which may be the state itself, while other segments may not have begun: they take
            // the given state from the scratch.
            if (seg == 0 && g.state != nullptr) {
                add(g.state + base, 1.f);
                store(p.local + local_base);
                #pragma unroll
                for (int c = 0; c < COLS; ++c)
                    #pragma unroll
                    for (int i = 0; i < ROWS / 2; ++i) S[c][i] = make_pair(0.f, 0.f);
            }
        } else {
            const float w0 = power(g2, (float)s0);
            if (g.state != nullptr) add(seg == 0 && last_seg ? g.state + base : p.local + local_base, w0);
            for (int x = 0; x < seg; ++x)
                add(p.local + local_base + (x + 1) * slice, power(g2, (float)((int64_t)(seg - 1 - x) * p.seg_len)));
        }
    }
    auto decay = [&](float l) {
        #pragma unroll
        for (int c = 0; c < COLS; ++c)
            #pragma unroll
            for (int i = 0; i < ROWS / 2; ++i) S[c][i] = mul_pair(S[c][i], make_pair(l, l));
    };
    if (threadIdx.x < kRecTile) {
        grow[threadIdx.x] = power(g2, -(float)threadIdx.x);             // (past the tile's length: not looked at)
        shrink[threadIdx.x] = power(g2, (float)threadIdx.x);
    }
    __syncthreads();
    // A tile's values on their way in registers while the tile before it is worked on: item i of a thread is token (128 i + thread) / DK,
    // element (128 i + thread) mod DK.
    constexpr int kPer = DK * kRecTile / kRecThreads, kPerV = DV * kRecTile / kRecThreads;
    T rq[kStates ? 1 : kPer], rk[kPer], rv[kPerV];
    auto fetch = [&](int64_t at, int n) {
        const T *qt = q + at * g.q_token, *kt = k + at * g.k_token, *vt = v + at * g.v_token;
        #pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int t = (i * kRecThreads + threadIdx.x) / DK, d = (i * kRecThreads + threadIdx.x) % DK;
            const bool ok = t < n && d < g.Dk;
            if constexpr (!kStates) rq[i] = ok ? qt[t * g.q_token + d] : from_f32<T>(0.f);
            rk[i] = ok ? kt[t * g.k_token + d] : from_f32<T>(0.f);
        }
        #pragma unroll
        for (int i = 0; i < kPerV; ++i) {
            const int t = (i * kRecThreads + threadIdx.x) / DV, c = (i * kRecThreads + threadIdx.x) % DV;
            rv[i] = t < n && c < cols ? vt[t * g.v_token + c] : from_f32<T>(0.f);
        }
    };
    int64_t t0 = 0;
    fetch(0, n_tok < tile ? (int)n_tok : tile);
    while (t0 < n_tok) {
        const int n = n_tok - t0 < tile ? (int)(n_tok - t0) : tile;
        #pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int t = (i * kRecThreads + threadIdx.x) / DK, d = (i * kRecThreads + threadIdx.x) % DK;
            if (t < n) {
                if constexpr (!kStates) sq[t][d] = to_f32(rq[i]) * shrink[t];
                sk[t][d] = to_f32(rk[i]) * grow[t];
            }
        }
        #pragma unroll
        for (int i = 0; i < kPerV; ++i) {
            const int t = (i * kRecThreads + threadIdx.x) / DV, c = (i * kRecThreads + threadIdx.x) % DV;
            if (t < n) sv[t][c] = to_f32(rv[i]);
        }
        const int64_t t1 = t0 + n;
        fetch(t1, n_tok - t1 < tile ? (int)(n_tok - t1) : tile);
        decay(power(g2, t0 == 0 ? 1.f : (float)tile));
        __syncthreads();
        for (int t = 0; t < n; ++t) {
            pair_t vt[COLS], o[COLS];
            #pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const float x = sv[t][lane + 32 * c];
                vt[c] = make_pair(x, x);
                o[c] = make_pair(0.f, 0.f);
            }
            const float4* k4 = reinterpret_cast<const float4*>(&sk[t][warp * ROWS]);
            const float4* q4 = reinterpret_cast<const float4*>(&sq[kStates ? 0 : t][warp * ROWS]);
            #pragma unroll
            for (int i = 0; i < ROWS / 4; ++i) {
                const float4 kk = k4[i];
                const pair_t ka = make_pair(kk.x, kk.y), kb = make_pair(kk.z, kk.w);
                #pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    S[c][2 * i] = fma_pair(ka, vt[c], S[c][2 * i]);
                    S[c][2 * i + 1] = fma_pair(kb, vt[c], S[c][2 * i + 1]);
                }
                if constexpr (!kStates) {
                    const float4 qq = q4[i];
                    const pair_t qa = make_pair(qq.x, qq.y), qb = make_pair(qq.z, qq.w);
                    #pragma unroll
                    for (int c = 0; c < COLS; ++c) {
                        o[c] = fma_pair(qa, S[c][2 * i], o[c]);
                        o[c] = fma_pair(qb, S[c][2 * i + 1], o[c]);
                    }
                }
            }
            if constexpr (!kStates) {
                #pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    float a, b2;
                    take_pair(o[c], a, b2);
                    so[t][warp][lane + 32 * c] = a + b2;
                }
            }
        }
        __syncthreads();
        if constexpr (!kStates) {
            for (int i = threadIdx.x; i < n * cols; i += kRecThreads) {
                const int t = i / cols, c = i % cols;
                const float o = (so[t][0][c] + so[t][1][c]) + (so[t][2][c] + so[t][3][c]);
                out[(t0 + t) * g.o_token + c] = from_f32<T>(g.scale * o);
            }
        }
        t0 += n;
        if (t0 >= n_tok) decay(power(g2, (float)(n - 1)));
    }
    if (kStates) store(p.local + local_base + (seg + 1) * slice);
    else if (last_seg) store(g.state_out + base);
}

template <typename T, int ROWS, int COLS>
cudaError_t launch_recurrent_rows(const DecayArgs& g, cudaStream_t s)
{
    const int slices = (g.Dv + COLS * 32 - 1) / (COLS * 32);
    // Few heads and long prompts: segments, until about four CTAs per SM walk a share of the tokens each; one launch finds what
    // each adds to the state, the next starts each from the decayed sum of what came before it.
    RecPlan p{};
    const int64_t ctas = g.B * g.H * slices;
    int64_t segs = 4 * (int64_t)device_sm_count() / ctas;
    if (segs > g.max_len / 128) segs = g.max_len / 128;
    if (segs > 16) segs = 16;
    if (segs < 1) segs = 1;
    p.seg_len = (g.max_len + segs - 1) / segs;
    if (p.seg_len < 1) p.seg_len = 1;
    p.segments = (int)((g.max_len + p.seg_len - 1) / p.seg_len);
    if (p.segments < 1) p.segments = 1;
    cudaError_t e = cudaSuccess;
    void* scratch = nullptr;
    if (p.segments > 1) {
        e = scratch_alloc(&scratch, (size_t)g.B * g.H * p.segments * g.Dk * g.Dv * sizeof(float), s);
        if (e != cudaSuccess) return e;
        p.local = static_cast<float*>(scratch);
        decay_recurrent_kernel<T, ROWS, COLS, true><<<dim3((unsigned)g.B, (unsigned)g.H, (unsigned)(slices * (p.segments - 1))), kRecThreads, 0, s>>>(g, p);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) {
        decay_recurrent_kernel<T, ROWS, COLS, false><<<dim3((unsigned)g.B, (unsigned)g.H, (unsigned)(slices * p.segments)), kRecThreads, 0, s>>>(g, p);
        e = cudaGetLastError();
    }
    if (scratch != nullptr) {
        const cudaError_t e2 = cudaFreeAsync(scratch, s);
        if (e == cudaSuccess) e = e2;
    }
    return e;
}

template <typename T>
cudaError_t launch_recurrent_typed(const DecayArgs& g, cudaStream_t s)
{
    if (g.Dk <= 64) return launch_recurrent_rows<T, 16, 2>(g, s);
    if (g.Dk <= 128) return launch_recurrent_rows<T, 32, 2>(g, s);
    return launch_recurrent_rows<T, 64, 1>(g, s);
}

}  // namespace

cudaError_t launch_decay_attention(const DecayArgs& g, cudaStream_t s)
{
    if (decay_chunk_supported(g)) {
        bool taken = false;
        const cudaError_t e = launch_decay_chunk(g, s, taken);
        if (taken) return e;
    }
    return with_dtype(g.dtype, [&](auto t) { return launch_recurrent_typed<decltype(t)>(g, s); });
}

cudaError_t launch_decay_attention_step(const DecayArgs& g, cudaStream_t s)
{
    return with_dtype(g.dtype, [&](auto t) { return launch_step_typed<decltype(t)>(g, s); });
}

}  // namespace rtn
