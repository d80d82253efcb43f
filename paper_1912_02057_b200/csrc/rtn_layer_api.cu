// C ABI of the layer operators (declared in rtn.h): argument checks and launches.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"

#include <limits.h>
#include <math.h>

namespace {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxK = int64_t(1) << 24;       // |S| <= K must stay exact in fp32 and int32
constexpr int64_t kMaxDim = int64_t(1) << 31;
constexpr int64_t kMaxStride = int64_t(1) << 40;

// Strides of a [tokens][heads][D] tensor: not negative, and no two elements in one place where it is written.
bool strides_ok(int64_t token, int64_t head) { return token >= 0 && head >= 0 && token < kMaxStride && head < kMaxStride; }
bool written_strides_ok(int64_t tokens, int64_t heads, int64_t D, int64_t token, int64_t head)
{
    if (!strides_ok(token, head)) return false;
    if (heads > 1 && head < D) return false;
    return tokens <= 1 || token >= (heads - 1) * head + D || (head >= (__int128)(tokens - 1) * token + D && token >= D);
}

rtn_status as_status(cudaError_t e) { return e == cudaSuccess ? RTN_OK : RTN_ERR_CUDA; }

// Checks common to the two attention entry points; fills everything but start, total and max_len.
rtn_status fill_decay(rtn::DecayArgs& g, const void* q, int64_t q_token, int64_t q_head, const void* k, int64_t k_token,
                      int64_t k_head, const void* v, int64_t v_token, int64_t v_head, void* out, int64_t o_token, int64_t o_head,
                      int64_t tokens, int64_t B, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, const float* log_decay, float scale,
                      const float* state, float* state_out, const int32_t* slots, int64_t n_slots, rtn_dtype dtype)
{
    if (log_decay == nullptr || (B > 0 && state_out == nullptr)) return RTN_ERR_NULL;
    if (tokens > 0 && (q == nullptr || k == nullptr || v == nullptr || out == nullptr)) return RTN_ERR_NULL;
    if (!rtn::dtype_ok(dtype)) return RTN_ERR_VALUE;
    if (H <= 0 || Hk <= 0 || H > 65535 || H % Hk != 0 || Dk <= 0 || Dv <= 0 || Dk > rtn::kDecayMaxDim || Dv > rtn::kDecayMaxDim)
        return RTN_ERR_SHAPE;
    if (n_slots < 0 || n_slots >= kMaxDim || (slots == nullptr && n_slots < B)) return RTN_ERR_SHAPE;
    if (!strides_ok(q_token, q_head) || !strides_ok(k_token, k_head) || !strides_ok(v_token, v_head) ||
        !written_strides_ok(tokens, H, Dv, o_token, o_head)) return RTN_ERR_SHAPE;
    const uintptr_t e = rtn::dtype_bytes(dtype);
    if (!aligned(q, e) || !aligned(k, e) || !aligned(v, e) || !aligned(out, e) || !aligned(log_decay, 4) || !aligned(state, 4) ||
        !aligned(state_out, 4) || !aligned(slots, 4)) return RTN_ERR_ALIGN;
    g.q = q; g.k = k; g.v = v;
    g.q_token = q_token; g.q_head = q_head; g.k_token = k_token; g.k_head = k_head; g.v_token = v_token; g.v_head = v_head;
    g.out = out; g.o_token = o_token; g.o_head = o_head;
    g.log_decay = log_decay; g.state = state; g.state_out = state_out; g.slot = slots; g.n_slots = n_slots;
    g.B = B; g.H = (int)H; g.Hk = (int)Hk; g.Dk = (int)Dk; g.Dv = (int)Dv; g.dtype = dtype; g.scale = scale;
    return RTN_OK;
}

}  // namespace

extern "C" {

rtn_status rtn_ternary_linear(const void* a_packed, const int32_t* a_sum, const void* w_packed, const int32_t* w_sum,
                              int64_t M, int64_t N, int64_t K, const float* a_scale, const float* a_offset, int64_t n_aparam,
                              const float* w_scale, const float* w_offset, int64_t n_wparam, const float* bias, rtn_activation act,
                              const void* residual, int64_t residual_stride, void* out, int64_t out_stride, rtn_dtype dtype, void* stream)
{
    if (w_packed == nullptr || w_sum == nullptr || w_scale == nullptr || w_offset == nullptr) return RTN_ERR_NULL;
    if (M > 0 && (a_packed == nullptr || a_sum == nullptr || a_scale == nullptr || a_offset == nullptr || out == nullptr)) return RTN_ERR_NULL;
    if (!rtn::dtype_ok(dtype) || (int)act < RTN_ACT_NONE || (int)act > RTN_ACT_SILU) return RTN_ERR_VALUE;
    if (M < 0 || N <= 0 || K <= 0 || M >= kMaxDim || N >= kMaxDim || K > kMaxK) return RTN_ERR_SHAPE;
    if ((n_aparam != 1 && n_aparam != M) || (n_wparam != 1 && n_wparam != N)) return RTN_ERR_SHAPE;
    if (out_stride < N || out_stride >= kMaxStride || (residual != nullptr && (residual_stride < 0 || residual_stride >= kMaxStride))) return RTN_ERR_SHAPE;
    if (residual == out && residual != nullptr && residual_stride != out_stride) return RTN_ERR_SHAPE;
    const uintptr_t e = rtn::dtype_bytes(dtype);
    if (!aligned(a_packed, 16) || !aligned(w_packed, 16) || !aligned(a_sum, 4) || !aligned(w_sum, 4) || !aligned(a_scale, 4) ||
        !aligned(a_offset, 4) || !aligned(w_scale, 4) || !aligned(w_offset, 4) || !aligned(bias, 4) || !aligned(residual, e) ||
        !aligned(out, e)) return RTN_ERR_ALIGN;
    if (M == 0) return RTN_OK;
    rtn::GemmArgs g{};
    g.a_packed = static_cast<const uint8_t*>(a_packed);
    g.a_sum = a_sum;
    g.w_packed = static_cast<const uint8_t*>(w_packed);
    g.w_sum = w_sum;
    g.M = M; g.N = N; g.K = K;
    g.ep = rtn::EpilogueParams{a_scale, a_offset, n_aparam, 0.f, 0.f, w_scale, w_offset, n_wparam};
    rtn::LinearArgs l{bias, (int)act, residual, residual_stride, out, out_stride, (int)dtype};
    if (rtn::linear_rows_path(M, N, K) && M > 8 * 65535) return RTN_ERR_UNSUPPORTED;
    g.status = rtn::device_status_word();
    if (g.status == nullptr) return RTN_ERR_CUDA;
    return as_status(rtn::launch_linear(g, l, static_cast<cudaStream_t>(stream)));
}

rtn_status rtn_rotary_table(float* table, int64_t rows, int64_t R, double base, rtn_rotary_scaling scaling, double factor,
                            double original_context, double low, double high, double amplitude, void* stream)
{
    if (table == nullptr) return RTN_ERR_NULL;
    if (rows <= 0 || rows >= (int64_t)INT_MAX * 256 || R < 2 || R % 2 != 0 || R > rtn::kRotaryMaxDim || rows * (R / 2) >= (int64_t)INT_MAX * 256) return RTN_ERR_SHAPE;
    if (!aligned(table, 4)) return RTN_ERR_ALIGN;
    if (!(base > 0.0) || !isfinite(base) || !isfinite(amplitude)) return RTN_ERR_VALUE;
    switch (scaling) {
        case RTN_ROTARY_SCALE_NONE: break;
        case RTN_ROTARY_SCALE_PARTS:
            if (!(original_context > 0.0) || !isfinite(original_context) || !(high > low) || !isfinite(high - low)) return RTN_ERR_VALUE;
            [[fallthrough]];
        case RTN_ROTARY_SCALE_LINEAR:
        case RTN_ROTARY_SCALE_BASE:
            if (!(factor > 0.0) || !isfinite(factor) || (scaling == RTN_ROTARY_SCALE_BASE && R <= 2)) return RTN_ERR_VALUE;
            break;
        default: return RTN_ERR_VALUE;
    }
    return as_status(rtn::launch_rotary_table(table, rows, (int)R, base, (int)scaling, factor, original_context, low, high, amplitude,
                                              static_cast<cudaStream_t>(stream)));
}

rtn_status rtn_qk_norm_rotary(const void* q, int64_t q_token, int64_t q_head, const void* k, int64_t k_token, int64_t k_head,
                              void* out_q, int64_t oq_token, int64_t oq_head, void* out_k, int64_t ok_token, int64_t ok_head,
                              int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t R, rtn_rotary_layout layout,
                              const float* q_weight, const float* k_weight, float eps, const float* table, int64_t table_rows,
                              const int64_t* positions, rtn_dtype dtype, void* stream)
{
    if (T < 0 || T >= kMaxDim || Hq <= 0 || Hk < 0 || D <= 0 || R < 0 || R > D || R % 2 != 0 || D > rtn::kRotaryMaxDim || Hq > 65535 || Hk > 65535 ||
        T * (Hq + Hk) >= (int64_t)INT_MAX || table_rows < 0) return RTN_ERR_SHAPE;
    if (T > 0 && (q == nullptr || out_q == nullptr || (Hk > 0 && (k == nullptr || out_k == nullptr)))) return RTN_ERR_NULL;
    if (R > 0 && (table == nullptr || table_rows == 0)) return RTN_ERR_NULL;
    if (q_weight == nullptr ? k_weight != nullptr : (Hk > 0 && k_weight == nullptr)) return RTN_ERR_NULL;
    if (!rtn::dtype_ok(dtype) || (layout != RTN_ROTARY_HALF && layout != RTN_ROTARY_INTERLEAVED)) return RTN_ERR_VALUE;
    if (q_weight != nullptr && !(eps >= 0.f)) return RTN_ERR_VALUE;
    if (!strides_ok(q_token, q_head) || !written_strides_ok(T, Hq, D, oq_token, oq_head)) return RTN_ERR_SHAPE;
    if (Hk > 0 && (!strides_ok(k_token, k_head) || !written_strides_ok(T, Hk, D, ok_token, ok_head))) return RTN_ERR_SHAPE;
    if (q == out_q && q != nullptr && (q_token != oq_token || q_head != oq_head)) return RTN_ERR_SHAPE;
    if (Hk > 0 && k == out_k && k != nullptr && (k_token != ok_token || k_head != ok_head)) return RTN_ERR_SHAPE;
    const uintptr_t e = rtn::dtype_bytes(dtype);
    if (!aligned(q, e) || !aligned(out_q, e) || (Hk > 0 && (!aligned(k, e) || !aligned(out_k, e))) || !aligned(q_weight, 4) ||
        !aligned(k_weight, 4) || !aligned(table, 4) || !aligned(positions, 8)) return RTN_ERR_ALIGN;
    if (T == 0) return RTN_OK;
    rtn::RotaryArgs g{};
    g.q = q; g.q_token = q_token; g.q_head = q_head;
    g.out_q = out_q; g.oq_token = oq_token; g.oq_head = oq_head;
    if (Hk > 0) {
        g.k = k; g.k_token = k_token; g.k_head = k_head;
        g.out_k = out_k; g.ok_token = ok_token; g.ok_head = ok_head;
    }
    g.q_weight = q_weight; g.k_weight = k_weight; g.eps = eps;
    g.table = table; g.table_rows = table_rows; g.positions = positions;
    g.T = T; g.Hq = (int)Hq; g.Hk = (int)Hk; g.D = (int)D; g.R = (int)R; g.layout = (int)layout; g.dtype = (int)dtype;
    g.status = rtn::device_status_word();
    if (g.status == nullptr) return RTN_ERR_CUDA;
    return as_status(rtn::launch_qk_norm_rotary(g, static_cast<cudaStream_t>(stream)));
}

rtn_status rtn_decay_attention(const void* q, int64_t q_token, int64_t q_head, const void* k, int64_t k_token, int64_t k_head,
                               const void* v, int64_t v_token, int64_t v_head, void* out, int64_t o_token, int64_t o_head,
                               int64_t total, int64_t B, const int32_t* start, int64_t max_len, int64_t H, int64_t Hk, int64_t Dk,
                               int64_t Dv, const float* log_decay, float scale, const float* state, float* state_out,
                               const int32_t* slots, int64_t n_slots, rtn_dtype dtype, void* stream)
{
    if (total < 0 || B < 0 || total >= kMaxDim || B >= kMaxDim || max_len < 0 || max_len >= kMaxDim) return RTN_ERR_SHAPE;
    if (start == nullptr) return RTN_ERR_NULL;
    if (!aligned(start, 4)) return RTN_ERR_ALIGN;
    rtn::DecayArgs g{};
    const rtn_status st = fill_decay(g, q, q_token, q_head, k, k_token, k_head, v, v_token, v_head, out, o_token, o_head, total, B, H,
                                     Hk, Dk, Dv, log_decay, scale, state, state_out, slots, n_slots, dtype);
    if (st != RTN_OK) return st;
    if (B == 0) return RTN_OK;
    g.start = start; g.total = total; g.max_len = max_len;
    g.status = rtn::device_status_word();
    if (g.status == nullptr) return RTN_ERR_CUDA;
    return as_status(rtn::launch_decay_attention(g, static_cast<cudaStream_t>(stream)));
}

rtn_status rtn_decay_attention_step(const void* q, int64_t q_token, int64_t q_head, const void* k, int64_t k_token, int64_t k_head,
                                    const void* v, int64_t v_token, int64_t v_head, void* out, int64_t o_token, int64_t o_head,
                                    int64_t B, int64_t H, int64_t Hk, int64_t Dk, int64_t Dv, const float* log_decay, float scale,
                                    const float* state, float* state_out, const int32_t* slots, int64_t n_slots, rtn_dtype dtype,
                                    void* stream)
{
    if (B < 0 || B >= kMaxDim || H <= 0 || H > 65535 || B * H >= (int64_t)INT_MAX / 8) return RTN_ERR_SHAPE;
    rtn::DecayArgs g{};
    const rtn_status st = fill_decay(g, q, q_token, q_head, k, k_token, k_head, v, v_token, v_head, out, o_token, o_head, B, B, H, Hk,
                                     Dk, Dv, log_decay, scale, state, state_out, slots, n_slots, dtype);
    if (st != RTN_OK) return st;
    if (B == 0) return RTN_OK;
    g.total = B; g.max_len = 1;
    g.status = rtn::device_status_word();
    if (g.status == nullptr) return RTN_ERR_CUDA;
    return as_status(rtn::launch_decay_attention_step(g, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
