// Linear attention with a decay l = exp(log_decay[h]) for each head h, per sequence and query head:
//
//   S_t = l S_{t-1} + k_t v_t^T        (S: Dk x Dv, fp32)
//   o_t = scale q_t^T S_t
//
// decay_step_kernel: one token per sequence.  Bound: DRAM, the fp32 state read and written once (8 Dk Dv bytes per head
//   against 4 Dk Dv operations).
// decay_recurrent_kernel: whole prompts token by token with the state in registers; any type, head dimension and
//   stride.  Bound: the FMA pipe (two FMAs and a product per state element and token).
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

constexpr int kRecCols = 32;            // state columns of a CTA, one per lane
constexpr int kRecWarps = 4;            // each holds a quarter of the rows
constexpr int kRecTile = 16;            // tokens staged at a time

template <typename T, int ROWS>
__global__ void __launch_bounds__(kRecCols * kRecWarps)
decay_recurrent_kernel(const DecayArgs g)
{
    constexpr int DK = ROWS * kRecWarps;
    __shared__ __align__(16) float sq[kRecTile][DK], sk[kRecTile][DK];
    __shared__ float sv[kRecTile][kRecCols], so[kRecTile][kRecWarps][kRecCols];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int h = blockIdx.y, hk = h / (g.H / g.Hk), c0 = blockIdx.z * kRecCols;
    const int64_t b = blockIdx.x;
    int64_t first, len, slot;
    if (!sequence_bounds(g, b, first, len, slot)) {
        if (threadIdx.x == 0) atomicOr(g.status, kStatusBadIndex);
        return;
    }
    const int cols = g.Dv - c0 < kRecCols ? g.Dv - c0 : kRecCols;
    T* out = static_cast<T*>(g.out) + first * g.o_token + h * g.o_head + c0;
    if (slot < 0) {
        for (int64_t i = threadIdx.x; i < len * cols; i += blockDim.x) out[(i / cols) * g.o_token + i % cols] = from_f32<T>(0.f);
        return;
    }
    const T* q = static_cast<const T*>(g.q) + first * g.q_token + h * g.q_head;
    const T* k = static_cast<const T*>(g.k) + first * g.k_token + hk * g.k_head;
    const T* v = static_cast<const T*>(g.v) + first * g.v_token + hk * g.v_head + c0;
    const float l = expf(g.log_decay[h]);
    const int64_t base = (slot * g.H + h) * (int64_t)g.Dk * g.Dv + c0 + lane;
    float S[ROWS];
    #pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = warp * ROWS + i;
        S[i] = g.state != nullptr && r < g.Dk && lane < cols ? g.state[base + (int64_t)r * g.Dv] : 0.f;
    }
    for (int64_t t0 = 0; t0 < len; t0 += kRecTile) {
        const int n = len - t0 < kRecTile ? (int)(len - t0) : kRecTile;
        for (int i = threadIdx.x; i < n * DK; i += blockDim.x) {
            const int t = i / DK, d = i % DK;
            sq[t][d] = d < g.Dk ? to_f32(q[(t0 + t) * g.q_token + d]) : 0.f;
            sk[t][d] = d < g.Dk ? to_f32(k[(t0 + t) * g.k_token + d]) : 0.f;
        }
        for (int i = threadIdx.x; i < n * kRecCols; i += blockDim.x) {
            const int t = i / kRecCols, c = i % kRecCols;
            sv[t][c] = c < cols ? to_f32(v[(t0 + t) * g.v_token + c]) : 0.f;
        }
        __syncthreads();
        for (int t = 0; t < n; ++t) {
            const float vt = sv[t][lane];
            const float4* k4 = reinterpret_cast<const float4*>(&sk[t][warp * ROWS]);
            const float4* q4 = reinterpret_cast<const float4*>(&sq[t][warp * ROWS]);
            float o0 = 0.f, o1 = 0.f;
            #pragma unroll
            for (int i = 0; i < ROWS / 4; ++i) {
                const float4 kk = k4[i], qq = q4[i];
                S[4 * i] = fmaf(l, S[4 * i], kk.x * vt);             o0 = fmaf(qq.x, S[4 * i], o0);
                S[4 * i + 1] = fmaf(l, S[4 * i + 1], kk.y * vt);     o1 = fmaf(qq.y, S[4 * i + 1], o1);
                S[4 * i + 2] = fmaf(l, S[4 * i + 2], kk.z * vt);     o0 = fmaf(qq.z, S[4 * i + 2], o0);
                S[4 * i + 3] = fmaf(l, S[4 * i + 3], kk.w * vt);     o1 = fmaf(qq.w, S[4 * i + 3], o1);
            }
            so[t][warp][lane] = o0 + o1;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n * cols; i += blockDim.x) {
            const int t = i / cols, c = i % cols;
            const float o = (so[t][0][c] + so[t][1][c]) + (so[t][2][c] + so[t][3][c]);
            out[(t0 + t) * g.o_token + c] = from_f32<T>(g.scale * o);
        }
        __syncthreads();
    }
    #pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = warp * ROWS + i;
        if (r < g.Dk && lane < cols) g.state_out[base + (int64_t)r * g.Dv] = S[i];
    }
}

template <typename T>
cudaError_t launch_recurrent_typed(const DecayArgs& g, cudaStream_t s)
{
    const dim3 grid((unsigned)g.B, (unsigned)g.H, (unsigned)((g.Dv + kRecCols - 1) / kRecCols));
    if (g.Dk <= 64) decay_recurrent_kernel<T, 16><<<grid, kRecCols * kRecWarps, 0, s>>>(g);
    else if (g.Dk <= 128) decay_recurrent_kernel<T, 32><<<grid, kRecCols * kRecWarps, 0, s>>>(g);
    else decay_recurrent_kernel<T, 64><<<grid, kRecCols * kRecWarps, 0, s>>>(g);
    return cudaGetLastError();
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
