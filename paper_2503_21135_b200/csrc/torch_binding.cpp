// Python calls of the operators around the layer on torch tensors: argument checks, result tensors, the current stream.  The
// arithmetic is all behind the C-ABI (include/dynamo.h).  A small call is bound by what the host does for it: through ctypes, with
// the same checks in Python, a combine of 64 tokens took 10.5 us and a gradient of the norm join 30, of which the launches are 3 and 5.
//
// A wrong tensor raises ValueError (one that requires a gradient while gradients are recorded as well), what the library refuses DynamoError; torch's own errors pass through.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/dynamo.h"

namespace {

using at::Tensor;

PyObject* g_dynamo_error = nullptr;   // the package's DynamoError

[[noreturn]] void refuse(const std::string& what) {
    PyErr_SetString(PyExc_ValueError, what.c_str());
    throw python_error();
}
void check_status(dynamo_status st, const char* where) {
    if (st == DYNAMO_OK) return;
    PyObject* e = PyObject_CallFunction(g_dynamo_error, "is", (int)st, where);
    if (e) {
        PyErr_SetObject(g_dynamo_error, e);
        Py_DECREF(e);
    }
    throw python_error();
}

// A launch can wait (a stream takes about a thousand), and what it waits for may be another Python thread or a callback: the interpreter's
// lock is given away for it, as torch's own calls do.  The arguments' tensors are held by the caller.
struct Unlocked {
    PyThreadState* const state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F>
dynamo_status unlocked(F f) {
    const Unlocked u;
    return f();
}

// Arguments arrive by position; None stands for what was left out.
struct Args {
    PyObject* const* v;
    Py_ssize_t n;
    Args(PyObject* const* args, Py_ssize_t given, Py_ssize_t wanted) : v(args), n(given) {
        if (given != wanted) refuse("internal: wrong number of arguments");
    }
    bool none(int i) const { return v[i] == Py_None; }
    const Tensor& tensor(int i, const char* name) const { return as_tensor(v[i], name); }
    static const Tensor& as_tensor(PyObject* o, const char* name) {
        if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor is wanted");
        return THPVariable_Unpack(o);
    }
    int64_t integer(int i, const char* name) const {
        const long long x = PyLong_AsLongLong(v[i]);
        if (x == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            refuse(std::string(name) + ": an integer is wanted");
        }
        return x;
    }
    bool truth(int i) const {
        const int t = PyObject_IsTrue(v[i]);
        if (t < 0) throw python_error();
        return t != 0;
    }
    float real(int i) const {
        const double x = PyFloat_AsDouble(v[i]);
        if (x == -1.0 && PyErr_Occurred()) throw python_error();
        return (float)x;
    }
};

int32_t size32(int64_t n, const char* name) {
    if (n > 0x7fffffff || n < -0x7fffffff) refuse(std::string(name) + ": too large");
    return (int32_t)n;
}
void on_cuda(const Tensor& t, const char* name) {
    if (!t.is_cuda() || t.layout() != at::kStrided) refuse(std::string(name) + ": a CUDA tensor is wanted");
}
void like(const Tensor& t, const char* name, c10::Device device) {
    // (results without a graph would leave such a tensor without its gradient, and nobody would be told)
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse(std::string(name) + ": its gradient is wanted, and this call records none (torch.no_grad() and the gradients' own calls)");
    if (t.layout() != at::kStrided || t.device() != device || !t.is_contiguous())
        refuse(std::string(name) + ": a contiguous tensor on " + device.str() + " is wanted");
}
void like(const Tensor& t, const char* name, c10::Device device, at::ScalarType type) {
    like(t, name, device);
    if (t.scalar_type() != type) refuse(std::string(name) + ": " + c10::toString(type) + " is wanted");
}
void shaped(const Tensor& t, const char* name, at::IntArrayRef shape) {
    if (t.sizes() == shape) return;
    std::string s;
    for (int64_t n : shape) s += (s.empty() ? "" : ", ") + std::to_string(n);
    refuse(std::string(name) + ": shape [" + s + "] is wanted");
}
int32_t type_code(const Tensor& t, const char* name) {
    if (t.scalar_type() == at::kBFloat16) return DYNAMO_BF16;
    if (t.scalar_type() == at::kFloat) return DYNAMO_F32;
    refuse(std::string(name) + ": bfloat16 or float32 is wanted");
}
at::ScalarType type_of(int64_t code, const char* name) {
    if (code == DYNAMO_BF16) return at::kBFloat16;
    if (code == DYNAMO_F32) return at::kFloat;
    refuse(std::string(name) + ": BF16 or F32 is wanted");
}
const void* ptr(const Tensor& t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void* mut(const Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
// (torch's own for the device: by way of its dispatcher an array takes some 0.2 us more)
Tensor empty(at::IntArrayRef shape, c10::Device device, at::ScalarType type) {
    return at::detail::empty_cuda(shape, type, device, std::nullopt);
}
// The tensors' device becomes the current one for the call, whose current stream takes the work.
struct OnDevice {
    c10::cuda::CUDAGuard guard;
    void* stream;
    explicit OnDevice(c10::Device d) : guard(d), stream((void*)c10::cuda::getCurrentCUDAStream(d.index()).stream()) {}
};
// A tensor of the caller's has been written: to automatic differentiation it is another now.  (Inference tensors count no versions, and
// nothing is kept of them.)
void written(const Tensor& t) {
    if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
PyObject* wrap(const Tensor& t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
template <typename... T>
PyObject* tuple_of(const T&... t) {
    PyObject* r = PyTuple_New(sizeof...(T));
    if (!r) throw python_error();
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(r, i++, wrap(t)), ...);
    return r;
}

// topk_idx, n_experts, x, out
PyObject* dispatch(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Args a(args, n, 4);
    const Tensor& idx = a.tensor(0, "topk_idx");
    on_cuda(idx, "topk_idx");
    const c10::Device device = idx.device();
    like(idx, "topk_idx", device, at::kInt);
    if (idx.dim() != 2) refuse("topk_idx: [T, k] is wanted");
    const int32_t T = size32(idx.size(0), "topk_idx"), k = size32(idx.size(1), "topk_idx"), E = size32(a.integer(1, "n_experts"), "n_experts");
    size_t need = 0;
    check_status(dynamo_dispatch_workspace_bytes(T, E, k, &need), "dynamo_dispatch_workspace_bytes");
    const bool with_x = !a.none(2);
    Tensor x, rows, offsets, perm, pos;
    int32_t d = 0, code = DYNAMO_BF16;
    if (with_x) {
        x = a.tensor(2, "x");
        like(x, "x", device);
        if (x.dim() != 2 || x.size(0) != T) refuse("x: [T, d] is wanted");
        d = size32(x.size(1), "x");
        code = type_code(x, "x");
    }
    const OnDevice on(device);
    const int64_t pairs = (int64_t)T * k;
    if (a.none(3)) {
        if (with_x) rows = empty({pairs, d}, device, x.scalar_type());
        offsets = empty({(int64_t)E + 1}, device, at::kInt);
        perm = empty({pairs}, device, at::kInt);
        pos = empty({T, k}, device, at::kInt);
    } else {
        if (!PyTuple_Check(args[3]) || PyTuple_GET_SIZE(args[3]) != 4) refuse("out: (rows, offsets, perm, pos) is wanted");
        PyObject* r = PyTuple_GET_ITEM(args[3], 0);
        if ((r == Py_None) == with_x) refuse("out.rows: given with x alone");
        if (with_x) {
            rows = Args::as_tensor(r, "out.rows");
            like(rows, "out.rows", device, x.scalar_type());
            shaped(rows, "out.rows", {pairs, d});
        }
        offsets = Args::as_tensor(PyTuple_GET_ITEM(args[3], 1), "out.offsets");
        perm = Args::as_tensor(PyTuple_GET_ITEM(args[3], 2), "out.perm");
        pos = Args::as_tensor(PyTuple_GET_ITEM(args[3], 3), "out.pos");
        like(offsets, "out.offsets", device, at::kInt);
        shaped(offsets, "out.offsets", {(int64_t)E + 1});
        like(perm, "out.perm", device, at::kInt);
        shaped(perm, "out.perm", {pairs});
        like(pos, "out.pos", device, at::kInt);
        shaped(pos, "out.pos", {T, k});
    }
    Tensor ws;
    if (need) ws = empty({(int64_t)need}, device, at::kByte);
    check_status(unlocked([&] {
        return dynamo_dispatch((const int32_t*)ptr(idx), T, E, k, ptr(x), d, code, (int32_t*)mut(offsets), (int32_t*)mut(perm),
                               (int32_t*)mut(pos), mut(rows), mut(ws), need, on.stream);
    }), "dynamo_dispatch");
    if (!a.none(3))
        for (const Tensor* t : {&rows, &offsets, &perm, &pos}) written(*t);
    return tuple_of(rows, offsets, perm, pos);
    END_HANDLE_TH_ERRORS
}

// rows and pos of a combine or its gradient
struct Routed {
    const Tensor &rows, &pos;
    Tensor w;
    c10::Device device;
    int32_t T, k, d, code;
    Routed(const Args& a, int rows_at, int pos_at, int w_at)
        : rows(a.tensor(rows_at, "rows")), pos(a.tensor(pos_at, "pos")), device((on_cuda(rows, "rows"), rows.device())) {
        like(rows, "rows", device);
        like(pos, "pos", device, at::kInt);
        if (rows.dim() != 2 || pos.dim() != 2 || rows.size(0) != pos.numel()) refuse("rows: [T k, d] and pos: [T, k] are wanted");
        T = size32(pos.size(0), "pos");
        k = size32(pos.size(1), "pos");
        d = size32(rows.size(1), "rows");
        code = type_code(rows, "rows");
        if (!a.none(w_at)) {
            w = a.tensor(w_at, "topk_w");
            like(w, "topk_w", device, at::kFloat);
            shaped(w, "topk_w", {T, k});
        }
    }
};

// rows, pos, topk_w, y_dtype, out
PyObject* combine(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Args a(args, n, 5);
    const Routed r(a, 0, 1, 2);
    const at::ScalarType y_type = a.none(3) ? r.rows.scalar_type() : type_of(a.integer(3, "y_dtype"), "y_dtype");
    const OnDevice on(r.device);
    Tensor y;
    if (a.none(4)) {
        y = empty({r.T, r.d}, r.device, y_type);
    } else {
        y = a.tensor(4, "out");
        like(y, "out", r.device, y_type);
        shaped(y, "out", {r.T, r.d});
    }
    const int32_t y_code = type_code(y, "out");
    check_status(unlocked([&] {
        return dynamo_combine(ptr(r.rows), r.code, (const int32_t*)ptr(r.pos), (const float*)ptr(r.w), r.T, r.k, r.d, mut(y),
                              y_code, on.stream);
    }), "dynamo_combine");
    if (!a.none(4)) written(y);
    return wrap(y);
    END_HANDLE_TH_ERRORS
}

// dy, rows, pos, topk_w, d_rows, want_d_w
PyObject* combine_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Args a(args, n, 6);
    const Routed r(a, 1, 2, 3);
    const Tensor& dy = a.tensor(0, "dy");
    like(dy, "dy", r.device);
    shaped(dy, "dy", {r.T, r.d});
    const int32_t dy_code = type_code(dy, "dy");
    const OnDevice on(r.device);
    Tensor d_rows, d_w;
    if (a.none(4)) {
        d_rows = empty(r.rows.sizes(), r.device, r.rows.scalar_type());
    } else {
        d_rows = a.tensor(4, "d_rows");
        like(d_rows, "d_rows", r.device, r.rows.scalar_type());
        shaped(d_rows, "d_rows", r.rows.sizes());
    }
    if (a.truth(5)) d_w = empty({r.T, r.k}, r.device, at::kFloat);
    check_status(unlocked([&] {
        return dynamo_combine_backward(ptr(dy), dy_code, ptr(r.rows), r.code, (const int32_t*)ptr(r.pos), (const float*)ptr(r.w),
                                       r.T, r.k, r.d, mut(d_rows), (float*)mut(d_w), on.stream);
    }), "dynamo_combine_backward");
    if (!a.none(4)) written(d_rows);
    return tuple_of(d_rows, d_w);
    END_HANDLE_TH_ERRORS
}

// What the two directions of the norm join have in common: r, y, w_post, gate, w_pre, post_norm, pre_norm, res_scale,
// block_scale, eps from argument `at` on.
struct Join {
    const Tensor& r;
    Tensor y, w_post, gate, w_pre;
    c10::Device device;
    int32_t T;
    dynamo_join_desc D;
    Join(const Args& a, int at, int32_t n_code) : r(a.tensor(at, "r")), device((on_cuda(r, "r"), r.device())) {
        like(r, "r", device);
        if (r.dim() != 2) refuse("r: [T, d] is wanted");
        T = size32(r.size(0), "r");
        D.d = size32(r.size(1), "r");
        D.r_dtype = D.y_dtype = type_code(r, "r");
        D.n_dtype = n_code;
        const bool post = a.truth(at + 5), pre = a.truth(at + 6);
        if (!a.none(at + 1)) {
            y = a.tensor(at + 1, "y");
            like(y, "y", device);
            shaped(y, "y", r.sizes());
            D.y_dtype = type_code(y, "y");
        } else if (!a.none(at + 2) || !a.none(at + 3)) {
            refuse("gate and w_post go with y");
        }
        if (!post && !a.none(at + 2)) refuse("w_post goes with post_norm");
        if (!pre && !a.none(at + 4)) refuse("w_pre goes with pre_norm");
        int32_t w_code = -1;
        auto weight = [&](int i, const char* name, Tensor& w) {
            w = a.tensor(i, name);
            like(w, name, device);
            shaped(w, name, {D.d});
            const int32_t code = type_code(w, name);
            if (w_code >= 0 && code != w_code) refuse("w_post, gate and w_pre: one type is wanted");
            w_code = code;
        };
        D.gate_kind = DYNAMO_GATE_NONE;
        if (!a.none(at + 3)) {
            gate = a.tensor(at + 3, "gate");
            if (gate.dim() == 2) {
                D.gate_kind = DYNAMO_GATE_TOKEN;
                like(gate, "gate", device, at::kFloat);
                shaped(gate, "gate ([d] or [T, 1])", {T, 1});
            } else {
                D.gate_kind = DYNAMO_GATE_CHANNEL;
                weight(at + 3, "gate ([d] or [T, 1])", gate);
            }
        }
        if (!a.none(at + 2)) weight(at + 2, "w_post", w_post);
        if (!a.none(at + 4)) weight(at + 4, "w_pre", w_pre);
        D.w_dtype = w_code < 0 ? DYNAMO_F32 : w_code;
        D.post_norm = post && y.defined();
        D.pre_norm = pre;
        D.res_scale = a.real(at + 7);
        D.block_scale = a.real(at + 8);
        D.eps = a.real(at + 9);
    }
};

// r, y, w_post, gate, w_pre, post_norm, pre_norm, res_scale, block_scale, eps, n_dtype, want_stats, r_out, n_out
PyObject* norm_join(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Args a(args, n, 14);
    const int64_t n_code = a.integer(10, "n_dtype");
    const at::ScalarType n_type = type_of(n_code, "n_dtype");
    const Join j(a, 0, (int32_t)n_code);
    const OnDevice on(j.device);
    Tensor r_out, n_out, stats;
    if (!j.y.defined()) {
        if (!a.none(12)) refuse("r_out goes with y");
    } else if (a.none(12)) {
        r_out = empty(j.r.sizes(), j.device, j.r.scalar_type());
    } else {
        r_out = a.tensor(12, "r_out");
        like(r_out, "r_out", j.device, j.r.scalar_type());
        shaped(r_out, "r_out", j.r.sizes());
    }
    if (!j.D.pre_norm) {
        if (!a.none(13)) refuse("n_out goes with pre_norm");
    } else if (a.none(13)) {
        n_out = empty(j.r.sizes(), j.device, n_type);
    } else {
        n_out = a.tensor(13, "n_out");
        like(n_out, "n_out", j.device, n_type);
        shaped(n_out, "n_out", j.r.sizes());
    }
    const bool want_stats = a.truth(11);
    if (want_stats) stats = empty({j.T, 2}, j.device, at::kFloat);
    check_status(unlocked([&] {
        return dynamo_norm_join_forward(&j.D, ptr(j.r), ptr(j.y), ptr(j.w_post), ptr(j.gate), ptr(j.w_pre), j.T, mut(r_out),
                                        mut(n_out), (float*)mut(stats), on.stream);
    }), "dynamo_norm_join_forward");
    if (!a.none(12)) written(r_out);
    if (!a.none(13)) written(n_out);
    PyObject* res = PyTuple_New(want_stats ? 3 : 2);
    if (!res) throw python_error();
    if (j.y.defined() && a.none(12)) {
        PyTuple_SET_ITEM(res, 0, wrap(r_out));
    } else {   // the caller's own object: r itself, or the buffer that it gave
        PyObject* own = j.y.defined() ? args[12] : args[0];
        Py_INCREF(own);
        PyTuple_SET_ITEM(res, 0, own);
    }
    PyTuple_SET_ITEM(res, 1, wrap(n_out));
    if (want_stats) PyTuple_SET_ITEM(res, 2, wrap(stats));
    return res;
    END_HANDLE_TH_ERRORS
}

// d_n, d_r_out, stats, r, y, w_post, gate, w_pre, post_norm, pre_norm, res_scale, block_scale, eps
// -> d_r, d_y, d_w_post, d_gate, d_w_pre
PyObject* norm_join_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Args a(args, n, 13);
    const bool pre = a.truth(9);
    if (a.none(0) == pre) refuse("d_n goes with pre_norm");
    if (a.none(0) && a.none(1)) refuse("d_r_out: wanted without pre_norm");
    Tensor d_n, d_ro;
    if (pre) d_n = a.tensor(0, "d_n");
    const Join j(a, 3, pre ? type_code(d_n, "d_n") : (int32_t)DYNAMO_BF16);
    if (pre) {
        like(d_n, "d_n", j.device);
        shaped(d_n, "d_n", j.r.sizes());
    }
    if (!a.none(1)) {
        d_ro = a.tensor(1, "d_r_out");
        like(d_ro, "d_r_out", j.device, j.r.scalar_type());
        shaped(d_ro, "d_r_out", j.r.sizes());
    }
    const Tensor& stats = a.tensor(2, "stats");
    like(stats, "stats", j.device, at::kFloat);
    shaped(stats, "stats", {j.T, 2});
    const OnDevice on(j.device);
    Tensor d_r = empty(j.r.sizes(), j.device, j.r.scalar_type()), d_y, d_w_post, d_gate, d_w_pre, ws;
    if (j.y.defined()) d_y = empty(j.r.sizes(), j.device, j.y.scalar_type());
    if (j.w_post.defined()) d_w_post = empty({j.D.d}, j.device, at::kFloat);
    if (j.gate.defined()) d_gate = empty(j.gate.sizes(), j.device, at::kFloat);
    if (j.w_pre.defined()) d_w_pre = empty({j.D.d}, j.device, at::kFloat);
    size_t need = 0;
    check_status(dynamo_norm_join_workspace_bytes(&j.D, j.T, &need), "dynamo_norm_join_workspace_bytes");
    if (d_w_post.defined() || d_w_pre.defined() || j.D.gate_kind == DYNAMO_GATE_CHANNEL) ws = empty({(int64_t)need}, j.device, at::kByte);
    else need = 0;
    check_status(unlocked([&] {
        return dynamo_norm_join_backward(&j.D, ptr(d_n), ptr(d_ro), ptr(j.r), ptr(j.y), (const float*)ptr(stats), ptr(j.w_post),
                                         ptr(j.gate), ptr(j.w_pre), j.T, mut(d_r), mut(d_y), (float*)mut(d_w_post),
                                         (float*)mut(d_gate), (float*)mut(d_w_pre), mut(ws), need, on.stream);
    }), "dynamo_norm_join_backward");
    return tuple_of(d_r, d_y, d_w_post, d_gate, d_w_pre);
    END_HANDLE_TH_ERRORS
}

// w, group_size
PyObject* quantize_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Args a(args, n, 2);
    const Tensor& w = a.tensor(0, "w");
    on_cuda(w, "w");
    like(w, "w", w.device(), at::kBFloat16);
    if (w.dim() != 2) refuse("w: [N, K] is wanted");
    const int64_t G = a.integer(1, "group_size");
    if ((G != 64 && G != 128) || w.size(1) % G) refuse("group_size: 64 or 128, a divisor of K, is wanted");
    const int32_t N = size32(w.size(0), "w"), K = size32(w.size(1), "w");
    const OnDevice on(w.device());
    Tensor codes = empty({N, K / 2}, w.device(), at::kByte), params = empty({N, K / G, 2}, w.device(), at::kHalf);
    check_status(unlocked([&] {
        return dynamo_linear_quantize(ptr(w), N, K, (int32_t)G, mut(codes), mut(params), on.stream);
    }), "dynamo_linear_quantize");
    return tuple_of(codes, params);
    END_HANDLE_TH_ERRORS
}

// x, codes, params, y_dtype, out
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Args a(args, n, 5);
    const Tensor &x = a.tensor(0, "x"), &codes = a.tensor(1, "codes"), &params = a.tensor(2, "params");
    on_cuda(x, "x");
    const c10::Device device = x.device();
    like(x, "x", device, at::kBFloat16);
    if (x.dim() != 2) refuse("x: [T, K] is wanted");
    like(params, "params", device, at::kHalf);
    const int32_t T = size32(x.size(0), "x"), K = size32(x.size(1), "x");
    if (params.dim() != 3 || params.size(2) != 2 || params.size(1) < 1 || K % params.size(1)) refuse("params: [N, K / group_size, 2] is wanted");
    const int32_t N = size32(params.size(0), "params"), G = K / (int32_t)params.size(1);
    like(codes, "codes", device, at::kByte);
    shaped(codes, "codes", {N, K / 2});
    const at::ScalarType y_type = type_of(a.integer(3, "y_dtype"), "y_dtype");
    const OnDevice on(device);
    Tensor y;
    if (a.none(4)) {
        y = empty({T, N}, device, y_type);
    } else {
        y = a.tensor(4, "out");
        like(y, "out", device, y_type);
        shaped(y, "out", {T, N});
    }
    size_t need = 0;
    check_status(dynamo_linear_workspace_bytes(T, N, K, G, &need), "dynamo_linear_workspace_bytes");
    Tensor ws;
    if (need) ws = empty({(int64_t)need}, device, at::kByte);
    const int32_t y_code = type_code(y, "out");
    check_status(unlocked([&] {
        return dynamo_linear_forward(ptr(x), T, N, K, G, ptr(codes), ptr(params), mut(y), y_code, mut(ws), need, on.stream);
    }), "dynamo_linear_forward");
    if (!a.none(4)) written(y);
    return wrap(y);
    END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls) {
    Py_XINCREF(cls);
    Py_XDECREF(g_dynamo_error);
    g_dynamo_error = cls;
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    {"dispatch", (PyCFunction)(void (*)())dispatch, METH_FASTCALL, nullptr},
    {"combine", (PyCFunction)(void (*)())combine, METH_FASTCALL, nullptr},
    {"combine_backward", (PyCFunction)(void (*)())combine_backward, METH_FASTCALL, nullptr},
    {"norm_join", (PyCFunction)(void (*)())norm_join, METH_FASTCALL, nullptr},
    {"norm_join_backward", (PyCFunction)(void (*)())norm_join_backward, METH_FASTCALL, nullptr},
    {"quantize_linear", (PyCFunction)(void (*)())quantize_linear, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)())linear, METH_FASTCALL, nullptr},
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&g_module); }
