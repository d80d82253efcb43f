// Linear attention with a decay l = exp(log_decay[h]) for each head h, per sequence and query head:
//
//   S_t = l S_{t-1} + k_t v_t^T        (S: Dk x Dv, fp32)
//   o_t = scale q_t^T S_t
//
// decay_step_kernel: one token per sequence.  Bound: DRAM, the fp32 state read and written once (8 Dk Dv bytes per head
//   against 4 Dk Dv operations).
//   96 sequences x 32 heads of 128 x 128: 62 us in a graph, 6.5 TB/s, a plain copy's rate.
// decay_recurrent_kernel: whole prompts token by token with the state in registers; any type, head dimension and
//   stride.  Bound: the FMA pipe (two FMAs per state element and token), behind a chain of about 280 clocks per token that two or
//   three CTAs per SM hide in part.  8 prompts of 2048 tokens, 32 heads of 128, fp16: 1310 us, 0.35 of that rate.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"
#include "rtn_decay.cuh"

namespace rtn {

namespace {

// ------------------------------------------------------------------------------------------------ single tokens

constexpr int kStepBatch = 8;           // state vectors a thread has in flight

// CTA = (sequence, head, slice of VW-element column groups).  Thread (r, c) owns columns VW c .. of the rows r, r + nr, ...:
// a warp reads whole sectors of consecutive rows, and every state element is touched once.
template <typename T, int VW, int kStepThreads>
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
    float s[kStepBatch][VW];
    auto load = [&](int r) {                // the rows r, r + nr, ... of a batch
        #pragma unroll
        for (int i = 0; i < kStepBatch; ++i) {
            const int row = r + i * nr;
            #pragma unroll
            for (int e = 0; e < VW; ++e) s[i][e] = 0.f;
            if (mine && g.state != nullptr && row < g.Dk) {
                const float* p = g.state + base + (int64_t)row * g.Dv;
                if constexpr (VW == 4) {
                    const float4 f = *reinterpret_cast<const float4*>(p);
                    s[i][0] = f.x; s[i][1] = f.y; s[i][2] = f.z; s[i][3] = f.w;
                } else s[i][0] = *p;
            }
        }
    };
    load(r0);                               // (on its way while q and k are: 238 sequences x 8 heads of 64: 16.3 us instead of 18.6)
    for (int i = threadIdx.x; i < g.Dk; i += kStepThreads) { sq[i] = to_f32(q[i]); sk[i] = to_f32(k[i]); }
    float vv[VW], acc[VW];
    #pragma unroll
    for (int e = 0; e < VW; ++e) { vv[e] = mine ? to_f32(v[c * VW + e]) : 0.f; acc[e] = 0.f; }
    const float l = expf(g.log_decay[h]);
    __syncthreads();
    for (int r = r0; mine && r < g.Dk; r += kStepBatch * nr) {
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
        if (r + kStepBatch * nr < g.Dk) load(r + kStepBatch * nr);
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
    // As many columns (whole 128-byte rows) per CTA as make one batch of 128 threads, fewer where there are few heads and SMs are left: 15
    // sequences x 32 heads of 128 in slices of 32 columns 13.2 us, 128 at once 14.7; 131 x 16 of 64 in slices of 32 15.8 us, 64 at once 13.0
    const int fit = 128 * kStepBatch * 4 / g.Dk / 32 * 32;
    const int slice = g.B * g.H < 2 * device_sm_count() || fit < 32 ? 32 : fit < kDecayMaxDim ? fit : kDecayMaxDim;
    const int slices = (g.Dv + slice - 1) / slice;
    const unsigned grid = (unsigned)(g.B * g.H * slices);
    // 64 x 64 states are one batch of 128 threads, larger ones take 256 (238 sequences x 8 heads of 64: 12.4 us instead of 16.3)
    const bool small = (int64_t)g.Dk * (g.Dv < slice ? g.Dv : slice) <= 128 * kStepBatch * 4;
    if (vec && small) decay_step_kernel<T, 4, 128><<<grid, 128, 0, s>>>(g, slice, slices);
    else if (vec) decay_step_kernel<T, 4, 256><<<grid, 256, 0, s>>>(g, slice, slices);
    else decay_step_kernel<T, 1, 256><<<grid, 256, 0, s>>>(g, slice, slices);
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------------------------ prompts, token by token

constexpr int kRecTile = 8;             // tokens staged at a time, at most

struct RecPlan {
    int64_t seg_len;        // tokens of a segment
    int segments;           // of the longest sequence
    float* local;           // [B][H][segments][Dk][Dv]: the state before the first segment, then what each but the last adds to it
};

// l^n from log2 l; n = 0 gives 1 for every l.
__device__ __forceinline__ float power(float g2, float n) { return n == 0.f ? 1.f : exp2f(n * g2); }

// Column(s) of the state in the lanes of each warp, ROWS rows of it in registers by pairs.  Within a run of tokens i = 0, 1, ... the state is kept
// relative to the run's first token,
//   S_i = l^i S'_i,   S'_i = S'_(i-1) + (l^-i k_i) v_i^T,   o_i = (l^i q_i)^T S'_i,
// which leaves one FMA per element for the update and one for the output, two elements to an instruction.  A run is a tile or a half,
// a quarter, an eighth of one, the longest whose l^-i stay at 2^8 or below: the range of k v and of q is then fp32's own but for eight
// powers of two.  What the steeper heads' extra products cost: 1310 us for 8 x 2048 tokens of 32 heads of 128, fp16, at log decays down to
// -0.79, 1342 at -1, 1390 at -3, 1477 at -8.
template <typename T, int ROWS, int COLS, int WARPS, bool kStates>
__global__ void __launch_bounds__(WARPS * 32, WARPS == 4 ? 3 : 2)         // (a fourth CTA of 4 warps: prompts of 9656 and 4828 tokens, heads of 64, 318 us instead of 256)
decay_recurrent_kernel(const DecayArgs g, const RecPlan p)
{
    constexpr int kRecThreads = WARPS * 32, DK = ROWS * WARPS, DV = COLS * 32;
    __shared__ __align__(16) float sq[kStates ? 1 : kRecTile][DK], sk[kRecTile][DK];
    __shared__ float sv[kRecTile][DV], so[kStates ? 1 : kRecTile][WARPS][DV];
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
    const float steep = fabsf(g2);
    const int run = steep <= 8.f / 7.f ? 8 : steep <= 8.f / 3.f ? 4 : steep <= 8.f ? 2 : 1;
    static_assert(kRecTile == 8, "runs");
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
    const float run_decay = power(g2, (float)run);
    auto decay = [&](float l) {
        #pragma unroll
        for (int c = 0; c < COLS; ++c)
            #pragma unroll
            for (int i = 0; i < ROWS / 2; ++i) S[c][i] = mul_pair(S[c][i], make_pair(l, l));
    };
    // A tile's values on their way in registers while the tile before it is worked on: a thread has one element of every kEveryK-th
    // token of q and k, and of every kEveryV-th of v.
    static_assert(kRecThreads % DK == 0 && kRecThreads % DV == 0 && kRecTile * DK % kRecThreads == 0 && kRecTile * DV % kRecThreads == 0, "shares");
    constexpr int kEveryK = kRecThreads / DK, kEveryV = kRecThreads / DV, kPer = kRecTile / kEveryK, kPerV = kRecTile / kEveryV;
    const int dk = threadIdx.x % DK, tk = threadIdx.x / DK, dv = threadIdx.x % DV, tv = threadIdx.x / DV;
    T rq[kStates ? 1 : kPer], rk[kPer], rv[kPerV];
    const T *qt = q + tk * g.q_token + dk, *kt = k + tk * g.k_token + dk, *vt_ = v + tv * g.v_token + dv;
    auto fetch = [&](int n) {               // the tile that the pointers are at
        const int nk = dk < g.Dk ? n - tk : 0, nv = dv < cols ? n - tv : 0;
        #pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if constexpr (!kStates) rq[i] = i * kEveryK < nk ? qt[i * kEveryK * g.q_token] : from_f32<T>(0.f);
            rk[i] = i * kEveryK < nk ? kt[i * kEveryK * g.k_token] : from_f32<T>(0.f);
        }
        #pragma unroll
        for (int i = 0; i < kPerV; ++i) rv[i] = i * kEveryV < nv ? vt_[i * kEveryV * g.v_token] : from_f32<T>(0.f);
        qt += n * g.q_token; kt += n * g.k_token; vt_ += n * g.v_token;
    };
    float own_grow[kPer], own_shrink[kStates ? 1 : kPer];
    #pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const float place = (float)((tk + i * kEveryK) & (run - 1));
        own_grow[i] = power(g2, -place);
        if constexpr (!kStates) own_shrink[i] = power(g2, place);
    }
    T* ot = out + tv * g.o_token + dv;
    int64_t t0 = 0;
    fetch(n_tok < kRecTile ? (int)n_tok : kRecTile);
    while (t0 < n_tok) {
        const int n = n_tok - t0 < kRecTile ? (int)(n_tok - t0) : kRecTile;
        #pragma unroll
        for (int i = 0; i < kPer; ++i) {                // (rows past the tile's length: not looked at)
            if constexpr (!kStates) sq[tk + i * kEveryK][dk] = to_f32(rq[i]) * own_shrink[i];
            sk[tk + i * kEveryK][dk] = to_f32(rk[i]) * own_grow[i];
        }
        #pragma unroll
        for (int i = 0; i < kPerV; ++i) sv[tv + i * kEveryV][dv] = to_f32(rv[i]);
        const int64_t t1 = t0 + n;
        fetch(n_tok - t1 < kRecTile ? (int)(n_tok - t1) : kRecTile);
        decay(t0 == 0 ? power(g2, 1.f) : run_decay);
        __syncthreads();
        auto token = [&](int t) {
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
        };
        if (run == kRecTile) {                          // (with the test in one loop for both: 1472 us instead of 1310, 8 x 2048 tokens of 32 heads of 128)
            for (int t = 0; t < n; ++t) token(t);
        } else {
            #pragma unroll 1
            for (int t = 0; t < n; ++t) {
                if (t > 0 && (t & (run - 1)) == 0) decay(run_decay);
                token(t);
            }
        }
        __syncthreads();
        if constexpr (!kStates) {
            #pragma unroll
            for (int i = 0; i < kPerV; ++i) {
                const int t = tv + i * kEveryV;
                if (t < n && dv < cols) {
                    float o = 0.f;
                    #pragma unroll
                    for (int w = 0; w < WARPS; ++w) o += so[t][w][dv];
                    ot[i * kEveryV * g.o_token] = from_f32<T>(g.scale * o);
                }
            }
            ot += n * g.o_token;
        }
        t0 += n;
        if (t0 >= n_tok) decay(power(g2, (float)((n - 1) & (run - 1))));
    }
    if (kStates) store(p.local + local_base + (seg + 1) * slice);
    else if (last_seg) store(g.state_out + base);
}

template <typename T, int ROWS, int COLS, int WARPS>
cudaError_t launch_recurrent_rows(const DecayArgs& g, cudaStream_t s)
{
    const int slices = (g.Dv + COLS * 32 - 1) / (COLS * 32);
    // Few heads and long prompts: segments, until about sixteen warps per SM walk a share of the tokens each; one launch finds what
    // each adds to the state (half of the work once more), the next starts each from the decayed sum of what came before it.  Two
    // segments do not make up for that where one CTA per head already has an SM (four prompts of 2048 to 4096 tokens, 16 heads of 128: 805 us, in two 861).
    RecPlan p{};
    const int64_t ctas = g.B * g.H * slices;
    int64_t segs = (16 / WARPS) * (int64_t)device_sm_count() / ctas;
    if (segs > g.max_len / 128) segs = g.max_len / 128;
    if (segs > 16) segs = 16;
    if (segs < 1 || (segs == 2 && 2 * ctas > device_sm_count())) segs = 1;
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
        decay_recurrent_kernel<T, ROWS, COLS, WARPS, true><<<dim3((unsigned)g.B, (unsigned)g.H, (unsigned)(slices * (p.segments - 1))), WARPS * 32, 0, s>>>(g, p);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) {
        decay_recurrent_kernel<T, ROWS, COLS, WARPS, false><<<dim3((unsigned)g.B, (unsigned)g.H, (unsigned)(slices * p.segments)), WARPS * 32, 0, s>>>(g, p);
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
    // 8 warps of 16 rows rather than 4 of 32: 128 registers hold them, 2594 -> 1743 us for 32768 tokens of 16 heads of 128
    if (g.Dk <= 64) return launch_recurrent_rows<T, 16, 2, 4>(g, s);
    if (g.Dk <= 128) return launch_recurrent_rows<T, 16, 2, 8>(g, s);
    return launch_recurrent_rows<T, 32, 2, 8>(g, s);
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
