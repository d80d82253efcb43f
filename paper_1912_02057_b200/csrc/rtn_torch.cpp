// Torch side of the layer operators: takes the tensors' addresses, shapes and strides, checks them, makes the outputs and calls the C
// ABI (rtn.h).  The ctypes marshalling of the other entry points costs 10 us for a call of this many tensors, several times what
// the kernels of a decoding step take; here it is one.
//
// The library's entry points come in by address (bind), so that whichever build of it the process has loaded is the one that is called.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include "rtn.h"

namespace {

decltype(&rtn_ternary_linear) f_linear;
decltype(&rtn_qk_norm_rotary) f_rotary;
decltype(&rtn_decay_attention) f_decay;
decltype(&rtn_decay_attention_step) f_step;
decltype(&rtn_packed_row_bytes) f_row_bytes;
decltype(&rtn_route_experts) f_route;
decltype(&rtn_ternary_experts) f_experts;
decltype(&rtn_block_norm) f_norm;
PyObject* rtn_error;                // class RtnError(code, where)
PyObject* torch_stream;             // class torch.cuda.Stream

// Thrown with the Python error already set.
struct Raised {};

[[noreturn]] void refuse(const std::string& what)
{
    PyErr_SetString(PyExc_ValueError, what.c_str());
    throw Raised{};
}

std::string text(const at::Tensor& t)
{
    std::string s = std::string(c10::toString(t.scalar_type())) + " [";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "] on " + t.device().str();
}

const at::Tensor* tensor_or_none(PyObject* o, const char* name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": expected a tensor");
    return &THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o, const char* name)
{
    const at::Tensor* t = tensor_or_none(o, name);
    if (t == nullptr) refuse(std::string(name) + ": a tensor is required");
    return *t;
}
int64_t whole(PyObject* o, const char* name)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    (void)name;
    return v;
}
double real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return v;
}

rtn_dtype type_of(at::ScalarType t)
{
    if (t == at::kFloat) return RTN_F32;
    if (t == at::kBFloat16) return RTN_BF16;
    if (t == at::kHalf) return RTN_F16;
    refuse(std::string("expected float32, bfloat16 or float16, got ") + c10::toString(t));
}

// The device of a call is that of its first tensor, and has to be the current one.
struct Call {
    c10::Device device;
    void* stream;
    bool given;                 // a stream of the caller's, not the current one
    bool lasting = false;       // one of torch's own, which are there as long as any tensor
    Call(const at::Tensor& first, PyObject* stream_or_none) : device(first.device()), given(stream_or_none != Py_None)
    {
        if (!first.is_cuda()) refuse("expected a CUDA tensor");
        const auto current = c10::cuda::current_device();
        if (device.index() != current) refuse("tensors on " + device.str() + ", but the current device is cuda:" + std::to_string(current));
        stream = c10::cuda::getCurrentCUDAStream(current).stream();
        if (!given) return;
        PyObject* handle = PyObject_GetAttrString(stream_or_none, "cuda_stream");
        if (handle == nullptr) throw Raised{};
        void* own = PyLong_AsVoidPtr(handle);
        Py_DECREF(handle);
        if (own == nullptr && PyErr_Occurred()) throw Raised{};
        lasting = own != stream && reinterpret_cast<PyObject*>(Py_TYPE(stream_or_none)) == torch_stream;
        stream = own;
    }
    // Memory that the call uses stays until its stream has: a temporary of the current stream, let go of when the call returns, would be given to the next
    // tensor there at once, and written while this stream is still to read it.  (An outside stream may be gone when a tensor is: its memory is the
    // caller's to keep.)
    void* use(const at::Tensor& t) const
    {
        if (lasting) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), device.index()));
        return t.data_ptr();
    }
    // A contiguous tensor of this type; None is NULL.
    template <typename T = void>
    T* dense(const at::Tensor* t, const char* name, at::ScalarType type, at::IntArrayRef shape = {}) const
    {
        if (t == nullptr) return nullptr;
        if (t->scalar_type() != type || t->device() != device || !t->is_contiguous() || (!shape.empty() && t->sizes() != shape)) {
            std::string want = c10::toString(type);
            if (!shape.empty()) { want += " ["; for (size_t i = 0; i < shape.size(); ++i) want += (i ? ", " : "") + std::to_string(shape[i]); want += "]"; }
            refuse(std::string(name) + ": expected contiguous " + want + " on " + device.str() + ", got " + text(*t));
        }
        return static_cast<T*>(use(*t));
    }
    // A result of the stream that writes it: on the current one's memory it could take the place of a tensor whose last use there
    // is still to come.
    at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) const
    {
        c10::cuda::OptionalCUDAStreamGuard on;
        if (given) on.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), device.index()));
        return at::detail::empty_cuda(shape, type, device, std::nullopt);
    }
};

// Address and strides of a [tokens, heads, D] tensor with adjacent elements.
struct Heads {
    void* p = nullptr;
    int64_t token = 0, head = 0;
    Heads() = default;
    Heads(const at::Tensor& t, const char* name, at::ScalarType type, const Call& call, int64_t T, int64_t H, int64_t D)
    {
        if (t.dim() != 3 || t.size(0) != T || t.size(1) != H || t.size(2) != D || t.scalar_type() != type || t.device() != call.device)
            refuse(std::string(name) + ": expected " + c10::toString(type) + " [" + std::to_string(T) + ", " + std::to_string(H) + ", " +
                   std::to_string(D) + "] on " + call.device.str() + ", got " + text(t));
        if (t.stride(2) != 1 && D > 1 && t.numel() > 0) refuse(std::string(name) + ": the elements of a head have to be adjacent");
        p = call.use(t); token = t.stride(0); head = t.stride(1);
    }
};

void check(rtn_status code, const char* where)
{
    if (code == RTN_OK) return;
    PyObject* e = PyObject_CallFunction(rtn_error, "is", (int)code, where);
    if (e != nullptr) { PyErr_SetObject(rtn_error, e); Py_DECREF(e); }
    throw Raised{};
}

void expect_args(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) { PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n); throw Raised{}; }
}

PyObject* pair_of(const at::Tensor& a, const at::Tensor* b)
{
    PyObject* x = THPVariable_Wrap(a);
    PyObject* y = b != nullptr ? THPVariable_Wrap(*b) : Py_NewRef(Py_None);
    PyObject* r = x != nullptr && y != nullptr ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return r;
}

// What dim 1 of a [tokens, heads, D] tensor must be asked before its shape is known to be one.
void want3(const at::Tensor& t, const char* name)
{
    if (t.dim() != 3) refuse(std::string(name) + ": expected [tokens, heads, D], got " + text(t));
}

// (scale, offset) of one operand: one value each or `full`.
int64_t params(const Call& call, const at::Tensor& scale, const at::Tensor& offset, int64_t full, const char* name, const float*& s, const float*& o)
{
    const int64_t n = scale.numel();
    if ((n != 1 && n != full) || offset.numel() != n)
        refuse(std::string(name) + "_scale and " + name + "_offset: expected 1 or " + std::to_string(full) + " values each, got " +
               std::to_string(n) + " and " + std::to_string(offset.numel()));
    s = call.dense<float>(&scale, name, at::kFloat);
    o = call.dense<float>(&offset, name, at::kFloat);
    return n;
}

// a_packed, a_sum, w_packed, w_sum, M, N, K, a_scale, a_offset, w_scale, w_offset, bias, activation, residual, out, dtype, stream
PyObject* linear(PyObject* const* a)
{
    const at::Tensor &ap = tensor(a[0], "a_packed"), &as = tensor(a[1], "a_sum"), &wp = tensor(a[2], "w_packed"), &ws = tensor(a[3], "w_sum");
    const int64_t M = whole(a[4], "M"), N = whole(a[5], "N"), K = whole(a[6], "K");
    const at::Tensor *bias = tensor_or_none(a[11], "bias"), *residual = tensor_or_none(a[13], "residual"), *given = tensor_or_none(a[14], "out");
    at::ScalarType type = at::kFloat;
    if (a[15] != Py_None) {
        if (!THPDtype_Check(a[15])) refuse("dtype: expected a torch.dtype");
        type = reinterpret_cast<THPDtype*>(a[15])->scalar_type;
    } else if (given != nullptr) type = given->scalar_type();
    else if (residual != nullptr) type = residual->scalar_type();
    const rtn_dtype dtype = type_of(type);
    const Call call(ap, a[16]);
    const int64_t row = (int64_t)f_row_bytes(K);
    if (M < 0 || N < 0 || ap.numel() < M * row || wp.numel() < N * row || as.numel() < M || ws.numel() < N)
        refuse("operands too small for M=" + std::to_string(M) + ", N=" + std::to_string(N) + ", K=" + std::to_string(K));
    const at::Tensor out = given != nullptr ? *given : call.empty({M, N}, type);
    void* at_[2] = {nullptr, nullptr};
    int64_t stride[2] = {0, 0};
    const at::Tensor* ends[2] = {residual, &out};
    for (int i = 0; i < 2; ++i) {
        const at::Tensor* t = ends[i];
        if (t == nullptr) continue;
        if (t->dim() != 2 || t->size(0) != M || t->size(1) != N || t->scalar_type() != type || t->device() != call.device || (t->stride(1) != 1 && N > 1))
            refuse(std::string(i ? "out" : "residual") + ": expected " + c10::toString(type) + " [" + std::to_string(M) + ", " + std::to_string(N) +
                   "] with adjacent columns on " + call.device.str() + ", got " + text(*t));
        at_[i] = call.use(*t);
        stride[i] = M > 1 ? t->stride(0) : std::max(N, t->stride(0));
    }
    const float *s1, *o1, *s2, *o2;
    const int64_t na = params(call, tensor(a[7], "a_scale"), tensor(a[8], "a_offset"), M, "a", s1, o1);
    const int64_t nw = params(call, tensor(a[9], "w_scale"), tensor(a[10], "w_offset"), N, "w", s2, o2);
    check(f_linear(call.dense(&ap, "a_packed", at::kByte), call.dense<int32_t>(&as, "a_sum", at::kInt), call.dense(&wp, "w_packed", at::kByte),
                   call.dense<int32_t>(&ws, "w_sum", at::kInt), M, N, K, s1, o1, na, s2, o2, nw, call.dense<float>(bias, "bias", at::kFloat, {N}),
                   (rtn_activation)whole(a[12], "activation"), at_[0], stride[0], at_[1], stride[1], dtype, call.stream), "rtn_ternary_linear");
    return given != nullptr ? Py_NewRef(a[14]) : THPVariable_Wrap(out);
}

// q, k, positions, table, q_weight, k_weight, eps, layout, out_q, out_k, stream
PyObject* rotary(PyObject* const* a)
{
    const at::Tensor& q = tensor(a[0], "q");
    const at::Tensor *k = tensor_or_none(a[1], "k"), *pos = tensor_or_none(a[2], "positions"), *table = tensor_or_none(a[3], "table");
    const at::Tensor *given_q = tensor_or_none(a[8], "out_q"), *given_k = tensor_or_none(a[9], "out_k");
    want3(q, "q");
    const at::ScalarType type = q.scalar_type();
    const rtn_dtype dtype = type_of(type);
    const Call call(q, a[10]);
    const int64_t T = q.size(0), Hq = q.size(1), D = q.size(2);
    const at::Tensor out_q = given_q != nullptr ? *given_q : call.empty({T, Hq, D}, type);
    const Heads hq(q, "q", type, call, T, Hq, D), oq(out_q, "out_q", type, call, T, Hq, D);
    int64_t Hk = 0;
    Heads hk, ok;
    at::Tensor out_k;
    if (k != nullptr) {
        want3(*k, "k");
        Hk = k->size(1);
        out_k = given_k != nullptr ? *given_k : call.empty({T, Hk, D}, type);
        hk = Heads(*k, "k", type, call, T, Hk, D);
        ok = Heads(out_k, "out_k", type, call, T, Hk, D);
    }
    if (table != nullptr && table->dim() != 2) refuse("table: expected [positions, R], got " + text(*table));
    const int64_t P = table != nullptr ? table->size(0) : 0, R = table != nullptr ? table->size(1) : 0;
    check(f_rotary(hq.p, hq.token, hq.head, hk.p, hk.token, hk.head, oq.p, oq.token, oq.head, ok.p, ok.token, ok.head, T, Hq, Hk, D, R,
                   (rtn_rotary_layout)whole(a[7], "layout"), call.dense<float>(tensor_or_none(a[4], "q_weight"), "q_weight", at::kFloat, {D}),
                   call.dense<float>(tensor_or_none(a[5], "k_weight"), "k_weight", at::kFloat, {D}), (float)real(a[6]),
                   call.dense<float>(table, "table", at::kFloat), P, call.dense<int64_t>(pos, "positions", at::kLong, {T}), dtype, call.stream),
          "rtn_qk_norm_rotary");
    return pair_of(out_q, k != nullptr ? &out_k : nullptr);
}

// What the two attention calls share.
struct Decay {
    Call call;
    int64_t T, H, Hk, Dk, Dv, slots_n;
    rtn_dtype dtype;
    at::Tensor out, state_out;
    Heads q, k, v, o;
    const float *log_decay, *state;
    float* after;
    const int32_t* slots;
    float scale;

    Decay(const at::Tensor& tq, const at::Tensor& tk, const at::Tensor& tv, const at::Tensor& g, const at::Tensor* given_state,
          const at::Tensor* given_after, const at::Tensor* given_slots, PyObject* given_scale, const at::Tensor* given_out, PyObject* stream, int64_t B)
        : call(tq, stream)
    {
        want3(tq, "q"); want3(tk, "k"); want3(tv, "v");
        const at::ScalarType type = tq.scalar_type();
        dtype = type_of(type);
        T = tq.size(0); H = tq.size(1); Dk = tq.size(2); Hk = tk.size(1); Dv = tv.size(2);
        if (B < 0) B = T;
        out = given_out != nullptr ? *given_out : call.empty({T, H, Dv}, type);
        if (given_after != nullptr) state_out = *given_after;
        else if (given_state != nullptr) state_out = *given_state;
        else if (given_slots != nullptr) refuse("slots without a state: state_out is required");
        else state_out = call.empty({B, H, Dk, Dv}, at::kFloat);
        if (state_out.dim() != 4) refuse("state_out: expected [slots, H, Dk, Dv], got " + text(state_out));
        slots_n = state_out.size(0);
        q = Heads(tq, "q", type, call, T, H, Dk);
        k = Heads(tk, "k", type, call, T, Hk, Dk);
        v = Heads(tv, "v", type, call, T, Hk, Dv);
        o = Heads(out, "out", type, call, T, H, Dv);
        log_decay = call.dense<float>(&g, "log_decay", at::kFloat, {H});
        state = call.dense<float>(given_state, "state", at::kFloat, {slots_n, H, Dk, Dv});
        after = call.dense<float>(&state_out, "state_out", at::kFloat, {slots_n, H, Dk, Dv});
        slots = call.dense<int32_t>(given_slots, "slots", at::kInt, {B});
        scale = given_scale == Py_None ? (float)(1.0 / std::sqrt((double)Dk)) : (float)real(given_scale);
    }
};

// q, k, v, log_decay, start, max_len, state, state_out, slots, scale, out, stream
PyObject* decay(PyObject* const* a)
{
    const at::Tensor& start = tensor(a[4], "start");
    if (start.dim() != 1 || start.numel() < 1) refuse("start: expected [B + 1], got " + text(start));
    const int64_t B = start.numel() - 1;
    const Decay d(tensor(a[0], "q"), tensor(a[1], "k"), tensor(a[2], "v"), tensor(a[3], "log_decay"), tensor_or_none(a[6], "state"),
                  tensor_or_none(a[7], "state_out"), tensor_or_none(a[8], "slots"), a[9], tensor_or_none(a[10], "out"), a[11], B);
    check(f_decay(d.q.p, d.q.token, d.q.head, d.k.p, d.k.token, d.k.head, d.v.p, d.v.token, d.v.head, d.o.p, d.o.token, d.o.head, d.T, B,
                  d.call.dense<int32_t>(&start, "start", at::kInt), whole(a[5], "max_len"), d.H, d.Hk, d.Dk, d.Dv, d.log_decay, d.scale,
                  d.state, d.after, d.slots, d.slots_n, d.dtype, d.call.stream), "rtn_decay_attention");
    return pair_of(d.out, &d.state_out);
}

// q, k, v, log_decay, state, state_out, slots, scale, out, stream
PyObject* step(PyObject* const* a)
{
    const Decay d(tensor(a[0], "q"), tensor(a[1], "k"), tensor(a[2], "v"), tensor(a[3], "log_decay"), tensor_or_none(a[4], "state"),
                  tensor_or_none(a[5], "state_out"), tensor_or_none(a[6], "slots"), a[7], tensor_or_none(a[8], "out"), a[9], -1);
    check(f_step(d.q.p, d.q.token, d.q.head, d.k.p, d.k.token, d.k.head, d.v.p, d.v.token, d.v.head, d.o.p, d.o.token, d.o.head, d.T, d.H, d.Hk,
                 d.Dk, d.Dv, d.log_decay, d.scale, d.state, d.after, d.slots, d.slots_n, d.dtype, d.call.stream), "rtn_decay_attention_step");
    return pair_of(d.out, &d.state_out);
}

// Address and row stride of a [rows, width] tensor with adjacent columns.
struct Rows {
    void* p = nullptr;
    int64_t stride = 0;
    Rows() = default;
    Rows(const at::Tensor& t, const char* name, at::ScalarType type, const Call& call, int64_t rows, int64_t width)
    {
        if (t.dim() != 2 || (rows >= 0 && t.size(0) != rows) || t.size(1) != width || t.scalar_type() != type || t.device() != call.device ||
            (t.stride(1) != 1 && width > 1 && t.size(0) > 0))
            refuse(std::string(name) + ": expected " + c10::toString(type) + " [" + (rows >= 0 ? std::to_string(rows) : "rows") + ", " +
                   std::to_string(width) + "] with adjacent columns on " + call.device.str() + ", got " + text(t));
        p = call.use(t);
        stride = t.size(0) > 1 ? t.stride(0) : std::max(width, t.stride(0));
    }
};

bool truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised{};
    return v != 0;
}

at::ScalarType dtype_of(PyObject* o, at::ScalarType otherwise)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) refuse("dtype: expected a torch.dtype");
    return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

PyObject* tuple_of(std::initializer_list<const at::Tensor*> ts)
{
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const at::Tensor* t : ts) {
        PyObject* x = t != nullptr && t->defined() ? THPVariable_Wrap(*t) : Py_NewRef(Py_None);
        if (r == nullptr || x == nullptr) { Py_XDECREF(r); Py_XDECREF(x); return nullptr; }
        PyTuple_SET_ITEM(r, i++, x);
    }
    return r;
}

// Thresholds and the places of the codes: none, or all of them.
struct Codes {
    const float *lo = nullptr, *hi = nullptr;
    int64_t n = 1;
    at::Tensor packed, sums;
    void* p = nullptr;
    int32_t* s = nullptr;
    Codes(const Call& call, PyObject* t_lo, PyObject* t_hi, PyObject* out_packed, PyObject* out_sum, int64_t rows, int64_t width, int64_t full)
    {
        const at::Tensor *a = tensor_or_none(t_lo, "t_lo"), *b = tensor_or_none(t_hi, "t_hi");
        const at::Tensor *gp = tensor_or_none(out_packed, "out_packed"), *gs = tensor_or_none(out_sum, "out_sum");
        if (a == nullptr && b == nullptr) {
            if (gp != nullptr || gs != nullptr) refuse("out_packed and out_sum: codes need t_lo and t_hi");
            return;
        }
        if (a == nullptr || b == nullptr) refuse("t_lo and t_hi: both, or neither");
        n = a->numel();
        if ((n != 1 && n != full) || b->numel() != n)
            refuse("t_lo and t_hi: expected 1 or " + std::to_string(full) + " values each, got " + std::to_string(n) + " and " + std::to_string(b->numel()));
        lo = call.dense<float>(a, "t_lo", at::kFloat);
        hi = call.dense<float>(b, "t_hi", at::kFloat);
        const int64_t row = (int64_t)f_row_bytes(width);
        packed = gp != nullptr ? *gp : call.empty({rows, row}, at::kByte);
        sums = gs != nullptr ? *gs : call.empty({rows}, at::kInt);
        p = call.dense(&packed, "out_packed", at::kByte, {rows, row});
        s = call.dense<int32_t>(&sums, "out_sum", at::kInt, {rows});
    }
};

// logits, top_k, score, bias, groups, kept_groups, group_top, renormalise, scale, plan, stream
PyObject* route(PyObject* const* a)
{
    const at::Tensor& logits = tensor(a[0], "logits");
    if (logits.dim() != 2) refuse("logits: expected [tokens, experts], got " + text(logits));
    const rtn_dtype dtype = type_of(logits.scalar_type());
    const Call call(logits, a[10]);
    const int64_t T = logits.size(0), E = logits.size(1), k = whole(a[1], "top_k"), groups = whole(a[4], "groups");
    if (k < 1 || k > 32) refuse("top_k: expected 1 to 32, got " + std::to_string(k));
    const Rows x(logits, "logits", logits.scalar_type(), call, T, E);
    const at::Tensor experts = call.empty({T, k}, at::kInt), weights = call.empty({T, k}, at::kFloat);
    at::Tensor start, tokens, place;
    const bool plan = truth(a[9]);
    if (plan) { start = call.empty({E + 1}, at::kInt); tokens = call.empty({T * k}, at::kInt); place = call.empty({T, k}, at::kInt); }
    auto at_ = [](const at::Tensor& t) { return t.defined() ? static_cast<int32_t*>(t.data_ptr()) : nullptr; };
    check(f_route(x.p, x.stride, T, E, dtype, (rtn_score)whole(a[2], "score"), call.dense<float>(tensor_or_none(a[3], "bias"), "bias", at::kFloat, {E}),
                  groups, a[5] == Py_None ? groups : whole(a[5], "kept_groups"), whole(a[6], "group_top"), k, truth(a[7]), (float)real(a[8]),
                  at_(experts), static_cast<float*>(weights.data_ptr()), at_(start), at_(tokens), at_(place), call.stream), "rtn_route_experts");
    return tuple_of({&experts, &weights, &start, &tokens, &place});
}

// a_packed, a_sum, tokens, start, w_packed, w_sum, N, K, a_scale, a_offset, w_scale, w_offset, bias, activation, gated, out, dtype, t_lo, t_hi,
// out_packed, out_sum, stream
PyObject* experts(PyObject* const* a)
{
    const at::Tensor &ap = tensor(a[0], "a_packed"), &as = tensor(a[1], "a_sum"), &start = tensor(a[3], "start");
    const at::Tensor &wp = tensor(a[4], "w_packed"), &ws = tensor(a[5], "w_sum");
    const at::Tensor *tokens = tensor_or_none(a[2], "tokens"), *bias = tensor_or_none(a[12], "bias"), *given = tensor_or_none(a[15], "out");
    const int64_t N = whole(a[6], "N"), K = whole(a[7], "K");
    const Call call(ap, a[21]);
    const bool gated = truth(a[14]);
    if (start.dim() != 1 || start.numel() < 2) refuse("start: expected [E + 1], got " + text(start));
    const int64_t E = start.numel() - 1, T = as.numel(), R = tokens != nullptr ? tokens->numel() : T, row = (int64_t)f_row_bytes(K);
    if (N <= 0 || K <= 0 || (gated && N % 2 != 0)) refuse("N and K: expected positive sizes (N even where gated), got " + std::to_string(N) + " and " + std::to_string(K));
    if (N > (INT64_C(1) << 31) / E || ap.numel() != T * row || wp.numel() != E * N * row || ws.numel() != E * N)
        refuse("operands do not fit E=" + std::to_string(E) + ", N=" + std::to_string(N) + ", K=" + std::to_string(K) + " and " + std::to_string(T) + " input rows");
    const int64_t F = gated ? N / 2 : N;
    const Codes codes(call, a[17], a[18], a[19], a[20], R, F, E);
    const at::ScalarType type = dtype_of(a[16], given != nullptr ? given->scalar_type() : at::kFloat);
    const rtn_dtype dtype = type_of(type);
    at::Tensor out;
    Rows o;
    if (given != nullptr || codes.p == nullptr) {
        out = given != nullptr ? *given : call.empty({R, F}, type);
        o = Rows(out, "out", type, call, R, F);
    }
    const float *s1, *o1, *s2, *o2;
    const int64_t na = params(call, tensor(a[8], "a_scale"), tensor(a[9], "a_offset"), T, "a", s1, o1);
    const int64_t nw = params(call, tensor(a[10], "w_scale"), tensor(a[11], "w_offset"), E * N, "w", s2, o2);
    if (bias != nullptr && bias->numel() != E * N) refuse("bias: expected " + std::to_string(E * N) + " values, got " + text(*bias));
    check(f_experts(call.dense(&ap, "a_packed", at::kByte), call.dense<int32_t>(&as, "a_sum", at::kInt), T,
                    call.dense<int32_t>(tokens, "tokens", at::kInt), call.dense<int32_t>(&start, "start", at::kInt), R, call.dense(&wp, "w_packed", at::kByte),
                    call.dense<int32_t>(&ws, "w_sum", at::kInt), E, N, K, s1, o1, na, s2, o2, nw, call.dense<float>(bias, "bias", at::kFloat),
                    (rtn_activation)whole(a[13], "activation"), gated, o.p, o.stride, dtype, codes.lo, codes.hi, codes.n, codes.p, codes.s, call.stream),
          "rtn_ternary_experts");
    if (!codes.packed.defined()) return given != nullptr ? Py_NewRef(a[15]) : THPVariable_Wrap(out);
    return tuple_of({&codes.packed, &codes.sums});
}

// branch, residual, place, weights, post_weight, gate, gate_kind, scale, norm_weight, eps, out, normed, t_lo, t_hi, out_packed, out_sum, dtype, stream
PyObject* block_norm(PyObject* const* a)
{
    const at::Tensor *branch = tensor_or_none(a[0], "branch"), *residual = tensor_or_none(a[1], "residual"), *place = tensor_or_none(a[2], "place");
    const at::Tensor *weights = tensor_or_none(a[3], "weights"), *gate = tensor_or_none(a[5], "gate"), *scale = tensor_or_none(a[7], "scale");
    const at::Tensor *given = tensor_or_none(a[10], "out"), *given_n = PyBool_Check(a[11]) ? nullptr : tensor_or_none(a[11], "normed");
    if (branch == nullptr && residual == nullptr) refuse("branch and residual: one of them is required");
    const at::Tensor& first = branch != nullptr ? *branch : *residual;
    const Call call(first, a[17]);
    if (first.dim() != 2) refuse("expected [rows, width], got " + text(first));
    const int64_t W = first.size(1), R = branch != nullptr ? branch->size(0) : 0;
    // (no choices: without this an empty place, which has no address, would be none, and row t what token t has)
    if (place != nullptr && (place->dim() != 2 || place->size(1) < 1)) refuse("place: expected [tokens, choices], got " + text(*place));
    const int64_t T = place != nullptr ? place->size(0) : first.size(0), k = place != nullptr ? place->size(1) : 0;
    const at::ScalarType stream_type = residual != nullptr ? residual->scalar_type() : given != nullptr ? given->scalar_type() : dtype_of(a[16], first.scalar_type());
    const at::ScalarType type = branch != nullptr ? branch->scalar_type() : given_n != nullptr ? given_n->scalar_type() : dtype_of(a[16], stream_type);
    const rtn_dtype dtype = type_of(type), stream_dtype = type_of(stream_type);
    Rows b, r, z, h, n;
    if (branch != nullptr) b = Rows(*branch, "branch", type, call, place != nullptr ? -1 : T, W);
    if (residual != nullptr) r = Rows(*residual, "residual", stream_type, call, T, W);
    if (gate != nullptr) z = Rows(*gate, "gate", type, call, T, W);
    const at::Tensor out = given != nullptr ? *given : call.empty({T, W}, stream_type);
    h = Rows(out, "out", stream_type, call, T, W);
    at::Tensor normed;
    if (given_n != nullptr || a[11] == Py_True) {
        normed = given_n != nullptr ? *given_n : call.empty({T, W}, type);
        n = Rows(normed, "normed", type, call, T, W);
    }
    const Codes codes(call, a[12], a[13], a[14], a[15], T, W, W);
    if (scale != nullptr && scale->numel() != 1 && scale->numel() != W) refuse("scale: expected 1 or " + std::to_string(W) + " values, got " + text(*scale));
    check(f_norm(b.p, b.stride, R, call.dense<int32_t>(place, "place", at::kInt), call.dense<float>(weights, "weights", at::kFloat, {T, k}), k,
                 call.dense<float>(tensor_or_none(a[4], "post_weight"), "post_weight", at::kFloat, {W}), z.p, z.stride, (rtn_gate)whole(a[6], "gate_kind"),
                 call.dense<float>(scale, "scale", at::kFloat), scale != nullptr ? scale->numel() : 1, r.p, r.stride,
                 call.dense<float>(tensor_or_none(a[8], "norm_weight"), "norm_weight", at::kFloat, {W}), (float)real(a[9]), T, W, h.p, h.stride,
                 n.p, n.stride, codes.lo, codes.hi, codes.n, codes.p, codes.s, dtype, stream_dtype, call.stream), "rtn_block_norm");
    return tuple_of({&out, &normed, &codes.packed, &codes.sums});
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    try {
        expect_args(n, N);
        return F(args);
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    try {
        expect_args(n, 10);
        f_linear = reinterpret_cast<decltype(f_linear)>(whole(args[0], ""));
        f_rotary = reinterpret_cast<decltype(f_rotary)>(whole(args[1], ""));
        f_decay = reinterpret_cast<decltype(f_decay)>(whole(args[2], ""));
        f_step = reinterpret_cast<decltype(f_step)>(whole(args[3], ""));
        f_row_bytes = reinterpret_cast<decltype(f_row_bytes)>(whole(args[4], ""));
        f_route = reinterpret_cast<decltype(f_route)>(whole(args[5], ""));
        f_experts = reinterpret_cast<decltype(f_experts)>(whole(args[6], ""));
        f_norm = reinterpret_cast<decltype(f_norm)>(whole(args[7], ""));
        rtn_error = Py_NewRef(args[8]);
        torch_stream = Py_NewRef(args[9]);
    } catch (const Raised&) {
        return nullptr;
    }
    Py_RETURN_NONE;
}

#define RTN_METHOD(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(static_cast<PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t)>(fn))), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RTN_METHOD("bind", bind), RTN_METHOD("linear", (entry<linear, 17>)), RTN_METHOD("rotary", (entry<rotary, 11>)),
                         RTN_METHOD("decay", (entry<decay, 12>)), RTN_METHOD("step", (entry<step, 10>)), RTN_METHOD("route", (entry<route, 11>)), RTN_METHOD("experts", (entry<experts, 22>)),
                         RTN_METHOD("block_norm", (entry<block_norm, 18>)), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rtn_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rtn_torch(void) { return PyModule_Create(&module); }
