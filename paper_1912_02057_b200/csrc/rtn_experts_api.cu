// C ABI of the operators of a layer of routed ternary experts (declared in rtn.h): argument checks and launches.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"

#include <limits.h>

namespace {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxK = int64_t(1) << 24;       // |S| <= K must stay exact in fp32 and int32
constexpr int64_t kMaxDim = int64_t(1) << 31;
constexpr int64_t kMaxStride = int64_t(1) << 40;

inline bool stride_ok(int64_t s) { return s >= 0 && s < kMaxStride; }
inline bool written_ok(int64_t s, int64_t width) { return s >= width && s < kMaxStride; }

rtn_status as_status(cudaError_t e) { return e == cudaSuccess ? RTN_OK : RTN_ERR_CUDA; }

}  // namespace

extern "C" {

rtn_status rtn_route_experts(const void* logits, int64_t logits_stride, int64_t T, int64_t E, rtn_dtype dtype, rtn_score score,
                             const float* bias, int64_t groups, int64_t kept_groups, int64_t group_top, int64_t top_k,
                             int renormalise, float weight_scale, int32_t* experts, float* weights,
                             int32_t* start, int32_t* tokens, int32_t* place, void* stream)
{
    if (T < 0 || E <= 0 || E > rtn::kMaxExperts || groups <= 0 || groups > rtn::kMaxChoices || E % groups != 0) return RTN_ERR_SHAPE;
    if (kept_groups <= 0 || kept_groups > groups || group_top <= 0 || group_top > E / groups) return RTN_ERR_SHAPE;
    if (top_k <= 0 || top_k > rtn::kMaxChoices || top_k > E / groups * kept_groups || T >= kMaxDim / top_k) return RTN_ERR_SHAPE;
    if (!rtn::dtype_ok(dtype) || (score != RTN_SCORE_SOFTMAX && score != RTN_SCORE_SIGMOID)) return RTN_ERR_VALUE;
    if (T > 1 ? !stride_ok(logits_stride) : logits_stride < 0) return RTN_ERR_SHAPE;
    if (T > 0 && (logits == nullptr || experts == nullptr || weights == nullptr)) return RTN_ERR_NULL;
    const bool plan = start != nullptr;
    if (plan ? T > 0 && (tokens == nullptr || place == nullptr) : tokens != nullptr || place != nullptr) return RTN_ERR_NULL;
    if (!aligned(logits, rtn::dtype_bytes(dtype)) || !aligned(bias, 4) || !aligned(experts, 4) || !aligned(weights, 4) || !aligned(start, 4) ||
        !aligned(tokens, 4) || !aligned(place, 4)) return RTN_ERR_ALIGN;
    if (T == 0 && !plan) return RTN_OK;
    rtn::RouteArgs g{};
    g.logits = logits; g.stride = logits_stride; g.T = T; g.E = (int)E; g.dtype = dtype; g.score = score; g.bias = bias;
    g.groups = (int)groups; g.kept = (int)kept_groups; g.group_top = (int)group_top; g.top_k = (int)top_k;
    g.renormalise = renormalise != 0; g.scale = weight_scale;
    g.experts = experts; g.weights = weights; g.start = start; g.tokens = tokens; g.place = place;
    return as_status(rtn::launch_route_experts(g, static_cast<cudaStream_t>(stream)));
}

rtn_status rtn_ternary_experts(const void* a_packed, const int32_t* a_sum, int64_t T, const int32_t* tokens, const int32_t* start, int64_t R,
                               const void* w_packed, const int32_t* w_sum, int64_t E, int64_t N, int64_t K,
                               const float* a_scale, const float* a_offset, int64_t n_aparam,
                               const float* w_scale, const float* w_offset, int64_t n_wparam, const float* bias,
                               rtn_activation act, int gated, void* out, int64_t out_stride, rtn_dtype dtype,
                               const float* t_lo, const float* t_hi, int64_t n_thr, void* out_packed, int32_t* out_sum, void* stream)
{
    if (T < 0 || R < 0 || T >= kMaxDim || R >= kMaxDim || E <= 0 || E > rtn::kMaxExperts || N <= 0 || N >= kMaxDim || K <= 0 || K > kMaxK ||
        E * N >= kMaxDim || (gated && N % 2 != 0)) return RTN_ERR_SHAPE;
    const int64_t F = gated ? N / 2 : N;
    if (tokens == nullptr && R > T) return RTN_ERR_SHAPE;
    if ((n_aparam != 1 && n_aparam != T) || (n_wparam != 1 && n_wparam != E * N)) return RTN_ERR_SHAPE;
    if (w_packed == nullptr || w_sum == nullptr || w_scale == nullptr || w_offset == nullptr || start == nullptr) return RTN_ERR_NULL;
    if (R > 0 && T > 0 && (a_packed == nullptr || a_sum == nullptr || a_scale == nullptr || a_offset == nullptr)) return RTN_ERR_NULL;
    const bool coded = out_packed != nullptr;
    if (coded ? out_sum == nullptr || t_lo == nullptr || t_hi == nullptr : out_sum != nullptr) return RTN_ERR_NULL;
    if (R > 0 && !coded && out == nullptr) return RTN_ERR_NULL;
    if (coded && n_thr != 1 && n_thr != E) return RTN_ERR_SHAPE;
    if (!rtn::dtype_ok(dtype) || (int)act < RTN_ACT_NONE || (int)act > RTN_ACT_SILU) return RTN_ERR_VALUE;
    if (out != nullptr && !written_ok(out_stride, F)) return RTN_ERR_SHAPE;
    if (!aligned(a_packed, 16) || !aligned(w_packed, 16) || !aligned(out_packed, 16) || !aligned(a_sum, 4) || !aligned(w_sum, 4) ||
        !aligned(tokens, 4) || !aligned(start, 4) || !aligned(a_scale, 4) || !aligned(a_offset, 4) || !aligned(w_scale, 4) ||
        !aligned(w_offset, 4) || !aligned(bias, 4) || !aligned(t_lo, 4) || !aligned(t_hi, 4) || !aligned(out_sum, 4) ||
        !aligned(out, rtn::dtype_bytes(dtype))) return RTN_ERR_ALIGN;
    if (R == 0) return RTN_OK;
    if (T == 0) return RTN_ERR_SHAPE;
    rtn::ExpertsArgs g{};
    g.a_packed = static_cast<const uint8_t*>(a_packed); g.a_sum = a_sum; g.T = T; g.tokens = tokens; g.start = start; g.R = R;
    g.w_packed = static_cast<const uint8_t*>(w_packed); g.w_sum = w_sum; g.E = (int)E; g.N = N; g.K = K; g.F = F;
    g.ep = rtn::EpilogueParams{a_scale, a_offset, n_aparam, 0.f, 0.f, w_scale, w_offset, n_wparam};
    g.bias = bias; g.act = (int)act; g.gated = gated != 0;
    g.out = out; g.out_stride = out_stride; g.dtype = dtype;
    g.t_lo = t_lo; g.t_hi = t_hi; g.n_thr = n_thr; g.out_packed = static_cast<uint8_t*>(out_packed); g.out_sum = out_sum;
    g.status = rtn::device_status_word();
    if (g.status == nullptr) return RTN_ERR_CUDA;
    return as_status(rtn::launch_ternary_experts(g, static_cast<cudaStream_t>(stream)));
}

rtn_status rtn_block_norm(const void* branch, int64_t branch_stride, int64_t R, const int32_t* place, const float* weights, int64_t k,
                          const float* post_weight, const void* gate, int64_t gate_stride, rtn_gate gate_kind,
                          const float* scale, int64_t n_scale, const void* residual, int64_t residual_stride,
                          const float* norm_weight, float eps, int64_t T, int64_t W, void* stream_out, int64_t stream_stride,
                          void* normed, int64_t normed_stride, const float* t_lo, const float* t_hi, int64_t n_thr,
                          void* out_packed, int32_t* out_sum, rtn_dtype dtype, rtn_dtype stream_dtype, void* stream)
{
    if (T < 0 || T >= kMaxDim || W <= 0 || W > rtn::kNormMaxWidth || R < 0 || R >= kMaxDim || k < 0 || k > rtn::kMaxChoices) return RTN_ERR_SHAPE;
    if ((place != nullptr) != (k > 0) && T > 0) return RTN_ERR_SHAPE;
    if (branch != nullptr && place == nullptr && R < T) return RTN_ERR_SHAPE;
    const bool none = branch == nullptr && !(place != nullptr && R == 0);           // (no rows: nothing to point at)
    if (T > 0 && none && residual == nullptr) return RTN_ERR_NULL;
    if (T > 0 && none && (place != nullptr || post_weight != nullptr || gate != nullptr || scale != nullptr)) return RTN_ERR_NULL;
    if (weights != nullptr && place == nullptr && T > 0) return RTN_ERR_NULL;
    const bool coded = out_packed != nullptr;
    if (coded ? out_sum == nullptr || t_lo == nullptr || t_hi == nullptr : out_sum != nullptr) return RTN_ERR_NULL;
    if (T > 0 && stream_out == nullptr && normed == nullptr && !coded) return RTN_ERR_NULL;
    if (coded && n_thr != 1 && n_thr != W) return RTN_ERR_SHAPE;
    if (scale != nullptr && n_scale != 1 && n_scale != W) return RTN_ERR_SHAPE;
    if (!rtn::dtype_ok(dtype) || !rtn::dtype_ok(stream_dtype) || (int)gate_kind < RTN_GATE_LINEAR || (int)gate_kind > RTN_GATE_SILU) return RTN_ERR_VALUE;
    if ((post_weight != nullptr || norm_weight != nullptr) && !(eps >= 0.f)) return RTN_ERR_VALUE;
    if ((branch != nullptr && !stride_ok(branch_stride)) || (gate != nullptr && !stride_ok(gate_stride)) ||
        (residual != nullptr && !stride_ok(residual_stride)) || (stream_out != nullptr && !written_ok(stream_stride, W)) ||
        (normed != nullptr && !written_ok(normed_stride, W))) return RTN_ERR_SHAPE;
    if (residual != nullptr && residual == stream_out && residual_stride != stream_stride) return RTN_ERR_SHAPE;
    const uintptr_t e = rtn::dtype_bytes(dtype), es = rtn::dtype_bytes(stream_dtype);
    if (!aligned(branch, e) || !aligned(gate, e) || !aligned(normed, e) || !aligned(residual, es) || !aligned(stream_out, es) ||
        !aligned(place, 4) || !aligned(weights, 4) || !aligned(post_weight, 4) || !aligned(scale, 4) || !aligned(norm_weight, 4) ||
        !aligned(t_lo, 4) || !aligned(t_hi, 4) || !aligned(out_sum, 4) || !aligned(out_packed, 16)) return RTN_ERR_ALIGN;
    if (T == 0) return RTN_OK;
    rtn::NormArgs g{};
    g.branch = branch; g.branch_stride = branch_stride; g.R = R; g.place = place; g.weights = weights; g.k = (int)k;
    g.post_weight = post_weight; g.gate = gate; g.gate_stride = gate_stride; g.gate_kind = gate_kind; g.scale = scale; g.n_scale = (int)n_scale;
    g.residual = residual; g.residual_stride = residual_stride; g.norm_weight = norm_weight; g.eps = eps; g.T = T; g.W = (int)W;
    g.stream_out = stream_out; g.stream_stride = stream_stride; g.normed = normed; g.normed_stride = normed_stride;
    g.t_lo = t_lo; g.t_hi = t_hi; g.n_thr = (int)n_thr; g.out_packed = static_cast<uint8_t*>(out_packed); g.out_sum = out_sum;
    g.dtype = dtype; g.stream_dtype = stream_dtype;
    g.status = rtn::device_status_word();
    if (g.status == nullptr) return RTN_ERR_CUDA;
    return as_status(rtn::launch_block_norm(g, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
