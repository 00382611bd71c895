// Native half of ops.py: checks tensors, allocates outputs and calls libef's entry points for the
// operators that make a worker's gradient.  A call through ctypes spends 16 us on the host for an
// RMS norm whose kernel takes 2; from here it spends half of that.  No arithmetic happens here, and the
// library is the one that the binding has loaded: its functions come in through bind().
#include <Python.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ef.h"

#include <optional>
#include <string>

namespace {

// ---- the library's functions -------------------------------------------------------------------
struct {
    decltype(&ef_checkpoint_save) checkpoint_save;
    decltype(&ef_checkpoint_load) checkpoint_load;
    decltype(&ef_rmsnorm_forward) rmsnorm_forward;
    decltype(&ef_rmsnorm_backward_workspace_bytes) rmsnorm_backward_workspace_bytes;
    decltype(&ef_rmsnorm_backward) rmsnorm_backward;
    decltype(&ef_activation_forward) activation_forward;
    decltype(&ef_activation_backward) activation_backward;
    decltype(&ef_checkpoint_weight_grad_workspace_bytes) checkpoint_weight_grad_workspace_bytes;
    decltype(&ef_checkpoint_weight_grad) checkpoint_weight_grad;
    decltype(&ef_token_logprob) token_logprob;
    decltype(&ef_policy_loss) policy_loss;
} lib = {};
PyObject* status_error = nullptr;                // called with (status, name): returns the exception to raise

struct Refused {};                               // a Python error is set

[[noreturn]] void refuse(const std::string& message) {
    PyErr_SetString(PyExc_ValueError, message.c_str());
    throw Refused{};
}
void check(int status, const char* name) {
    if (status == EF_OK) return;
    if (PyObject* e = PyObject_CallFunction(status_error, "is", status, name)) {
        PyErr_SetObject((PyObject*)Py_TYPE(e), e);
        Py_DECREF(e);
    }
    throw Refused{};
}

// ---- arguments ---------------------------------------------------------------------------------
const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor is needed");
    return THPVariable_Unpack(o);
}
const at::Tensor* optional_tensor(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

int type_of(at::ScalarType t) {
    return t == at::kFloat ? EF_TYPE_F32 : t == at::kBFloat16 ? EF_TYPE_BF16 : t == at::kHalf ? EF_TYPE_F16 : -1;
}

struct Matrix {
    const at::Tensor& t;
    int64_t n, c, ld;
    int type;
    void* p() const { return t.data_ptr(); }
};
// A CUDA matrix of a known type with neighbouring columns; of `like`'s rows, type and device, and of
// `cols` columns, where given.
Matrix matrix(const at::Tensor& t, const char* name, const Matrix* like = nullptr, int64_t cols = 0) {
    const int type = type_of(t.scalar_type());
    if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 2 || type < 0)
        refuse(std::string(name) + ": a CUDA matrix of float32, bfloat16 or float16 is needed");
    const int64_t n = t.size(0), c = t.size(1), ld = n > 1 ? t.stride(0) : c;
    if (c < 1 || ld < c || (t.stride(1) != 1 && c > 1))
        refuse(std::string(name) + ": a matrix with neighbouring columns, and at least one, is needed");
    if (like && (type != like->type || n != like->n || t.device() != like->t.device()))
        refuse(std::string(name) + ": type, rows or device differ");
    if (cols && c != cols)
        refuse(std::string(name) + ": " + std::to_string(cols) + " columns are needed, got " + std::to_string(c));
    return Matrix{t, n, c, ld, type};
}
Matrix matrix(PyObject* o, const char* name, const Matrix* like = nullptr, int64_t cols = 0) {
    return matrix(tensor(o, name), name, like, cols);
}
void* vec(PyObject* o, int64_t n, const char* name, const Matrix& like, at::ScalarType type = at::kFloat) {
    const at::Tensor& t = tensor(o, name);
    if (t.dim() != 1 || t.size(0) != n || t.scalar_type() != type || t.device() != like.t.device() || !t.is_contiguous())
        refuse(std::string(name) + ": a contiguous vector of " + std::to_string(n) + " of the right type and device is needed");
    return t.data_ptr();
}
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused{};
    return v != 0;
}
// A checkpoint as ops.Checkpoint describes it: rows, columns, and its codes and scales, or one buffer with both and None.
// The addresses are those of the tensors at this call: they may have been copied or unpickled since.
struct Kept {
    int64_t rows, cols;
    int device;
    int8_t* codes;
    float* scales;
};
Kept kept(PyObject* const* a) {
    const int64_t n = integer(a[0]), c = integer(a[1]);
    const at::Tensor& first = tensor(a[2], "checkpoint");
    const at::Tensor* const scales = optional_tensor(a[3], "checkpoint");
    auto holds = [](const at::Tensor& t, at::ScalarType type, int64_t count) {
        return t.is_cuda() && t.scalar_type() == type && t.is_contiguous() && t.numel() == count;
    };
    const int64_t codes = n * EF_CHECKPOINT_PITCH(c), groups = n * EF_CHECKPOINT_GROUPS(c);
    if (n < 0 || c < 1 || !holds(first, at::kChar, scales ? codes : codes + 4 * groups) ||
        (scales && (!holds(*scales, at::kFloat, groups) || scales->device() != first.device())))
        refuse("checkpoint: its codes and scales are not on a CUDA device, or not of its size");
    int8_t* const p = (int8_t*)first.data_ptr();
    return Kept{n, c, (int)first.get_device(), p, scales ? (float*)scales->data_ptr() : (float*)(p + codes)};
}

// ---- results -----------------------------------------------------------------------------------
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, c10::Device device) {
    return at::empty(sizes, at::TensorOptions().dtype(type).device(device));
}
// One buffer for a checkpoint: codes, then scales (the pitch is a multiple of 16 bytes).
at::Tensor fresh_checkpoint(int64_t n, int64_t c, c10::Device device) {
    return fresh({n * EF_CHECKPOINT_PITCH(c) + 4 * n * EF_CHECKPOINT_GROUPS(c)}, at::kChar, device);
}
int8_t* codes_of(const at::Tensor& t) { return t.defined() ? (int8_t*)t.data_ptr() : nullptr; }
float* scales_of(const at::Tensor& t, int64_t n, int64_t c) {
    return t.defined() ? (float*)((char*)t.data_ptr() + n * EF_CHECKPOINT_PITCH(c)) : nullptr;
}
// As torch does, a leaf that requires gradients, or a view of one, is not overwritten while gradients are recorded.
void check_overwritable(const at::Tensor& t, const char* name) {
    if (at::GradMode::is_enabled() && t.requires_grad() && (t.is_leaf() || (t.is_view() && t._base().is_leaf())))
        refuse(std::string(name) + ": a leaf that requires gradients would be overwritten");
}
// The library wrote to a tensor of the caller's: a backward pass that has saved its old values must notice.
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
PyObject* wrapped(at::Tensor t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(t));
}
template <class... T>
PyObject* pack(T... t) {
    PyObject* const tuple = PyTuple_New(sizeof...(T));
    if (!tuple) throw Refused{};
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(tuple, i++, wrapped(std::move(t))), ...);
    return tuple;
}

// The tensor's device made current, and its current stream.
struct On {
    c10::cuda::OptionalCUDAGuard guard;
    void* stream;
    explicit On(c10::Device d) {
        if (d.index() != c10::cuda::current_device()) guard.set_device(d);
        stream = c10::cuda::getCurrentCUDAStream(d.index()).stream();
    }
};

// ---- calls -------------------------------------------------------------------------------------
PyObject* checkpoint_save(PyObject* const* a) {
    const Matrix x = matrix(a[0], "x");
    at::Tensor b = fresh_checkpoint(x.n, x.c, x.t.device());
    const On on(x.t.device());
    check(lib.checkpoint_save(x.type, x.n, x.c, x.p(), x.ld, codes_of(b), scales_of(b, x.n, x.c), on.stream), "ef_checkpoint_save");
    return wrapped(std::move(b));
}

PyObject* checkpoint_load(PyObject* const* a) {
    const Kept k = kept(a);
    const int type = (int)integer(a[4]);
    const c10::Device device(c10::kCUDA, (c10::DeviceIndex)k.device);
    at::Tensor x = fresh({k.rows, k.cols}, type == EF_TYPE_F32 ? at::kFloat : type == EF_TYPE_BF16 ? at::kBFloat16 : at::kHalf, device);
    const On on(device);
    check(lib.checkpoint_load(type, k.rows, k.cols, k.codes, k.scales, x.data_ptr(), k.cols, on.stream), "ef_checkpoint_load");
    return wrapped(std::move(x));
}

PyObject* rmsnorm_forward(PyObject* const* a) {          // x, weight, eps, residual, checkpoint -> h, y, rstd, buffer
    const Matrix x = matrix(a[0], "x");
    const float* const w = (const float*)vec(a[1], x.c, "weight", x);
    const float eps = (float)number(a[2]);
    const at::Tensor* const res = optional_tensor(a[3], "residual");
    const c10::Device device = x.t.device();
    std::optional<Matrix> r;
    at::Tensor h, b;
    if (res) {
        r.emplace(matrix(*res, "residual", &x, x.c));
        h = fresh({x.n, x.c}, x.t.scalar_type(), device);
    }
    at::Tensor y = fresh({x.n, x.c}, x.t.scalar_type(), device), rstd = fresh({x.n}, at::kFloat, device);
    if (truth(a[4])) b = fresh_checkpoint(x.n, x.c, device);
    const On on(device);
    check(lib.rmsnorm_forward(x.type, x.n, x.c, x.p(), x.ld, r ? r->p() : nullptr, r ? r->ld : 0, w, eps,
                              h.defined() ? h.data_ptr() : nullptr, x.c, y.data_ptr(), x.c, (float*)rstd.data_ptr(),
                              codes_of(b), scales_of(b, x.n, x.c), on.stream), "ef_rmsnorm_forward");
    return pack(std::move(h), std::move(y), std::move(rstd), std::move(b));
}

PyObject* rmsnorm_backward(PyObject* const* a) {         // dy, h or None, its checkpoint (4), weight, rstd, dh -> dx, dw
    const Matrix dy = matrix(a[0], "dy");
    const at::Tensor* const ht = optional_tensor(a[1], "h");
    const float* const w = (const float*)vec(a[6], dy.c, "weight", dy);
    const float* const rstd = (const float*)vec(a[7], dy.n, "rstd", dy);
    const at::Tensor* const dht = optional_tensor(a[8], "dh");
    const c10::Device device = dy.t.device();
    std::optional<Matrix> h, dh;
    Kept k = {};
    if (ht) h.emplace(matrix(*ht, "h", &dy, dy.c));
    else {
        k = kept(a + 2);
        if (k.rows != dy.n || k.cols != dy.c || k.device != device.index()) refuse("h: a checkpoint of dy's shape is needed");
    }
    if (dht) dh.emplace(matrix(*dht, "dh", &dy, dy.c));
    at::Tensor dx = fresh({dy.n, dy.c}, dy.t.scalar_type(), device), dw = fresh({dy.c}, at::kFloat, device);
    size_t bytes = 0;
    check(lib.rmsnorm_backward_workspace_bytes(dy.n, dy.c, &bytes), "ef_rmsnorm_backward_workspace_bytes");
    const at::Tensor work = fresh({(int64_t)bytes}, at::kByte, device);
    const On on(device);
    check(lib.rmsnorm_backward(dy.type, dy.n, dy.c, dy.p(), dy.ld, h ? h->p() : nullptr, h ? h->ld : dy.c, k.codes, k.scales, w,
                               rstd, dh ? dh->p() : nullptr, dh ? dh->ld : 0, dx.data_ptr(), dy.c, (float*)dw.data_ptr(),
                               work.data_ptr(), bytes, on.stream), "ef_rmsnorm_backward");
    return pack(std::move(dx), std::move(dw));
}

PyObject* activation_forward(PyObject* const* a) {       // z, kind, checkpoint, checkpoint_out -> a, buffer of z, buffer of a
    const Matrix z = matrix(a[0], "z");
    const int kind = (int)integer(a[1]), parts = kind == EF_ACT_SWIGLU ? 2 : 1;
    const int64_t c = z.c / parts;
    if (c < 1 || z.c != c * parts) refuse("z: swiglu needs an even number of columns");
    const c10::Device device = z.t.device();
    at::Tensor out = fresh({z.n, c}, z.t.scalar_type(), device), bz, ba;
    if (truth(a[2])) bz = fresh_checkpoint(z.n * parts, c, device);
    if (truth(a[3])) ba = fresh_checkpoint(z.n, c, device);
    const On on(device);
    check(lib.activation_forward(z.type, kind, z.n, c, z.p(), z.ld, out.data_ptr(), c, codes_of(bz),
                                 scales_of(bz, z.n * parts, c), codes_of(ba), scales_of(ba, z.n, c), on.stream),
          "ef_activation_forward");
    return pack(std::move(out), std::move(bz), std::move(ba));
}

PyObject* activation_backward(PyObject* const* a) {      // da, kind, checkpoint of z (4) -> dz
    const Matrix da = matrix(a[0], "da");
    const int kind = (int)integer(a[1]), parts = kind == EF_ACT_SWIGLU ? 2 : 1;
    const Kept k = kept(a + 2);
    const c10::Device device = da.t.device();
    if (k.rows != da.n * parts || k.cols != da.c || k.device != device.index())
        refuse("z: the checkpoint does not belong to da's shape");
    at::Tensor dz = fresh({da.n, da.c * parts}, da.t.scalar_type(), device);
    const On on(device);
    check(lib.activation_backward(da.type, kind, da.n, da.c, da.p(), da.ld, k.codes, k.scales, dz.data_ptr(), da.c * parts,
                                  on.stream), "ef_activation_backward");
    return wrapped(std::move(dz));
}

PyObject* checkpoint_weight_grad(PyObject* const* a) {   // checkpoint of x (4), dy, out or None, accumulate -> out
    const Kept k = kept(a);
    const Matrix dy = matrix(a[4], "dy");
    const at::Tensor* const given = optional_tensor(a[5], "out");
    const bool accumulate = truth(a[6]);
    if (given) check_overwritable(*given, "out");
    const c10::Device device = dy.t.device();
    if (k.rows != dy.n || k.device != device.index()) refuse("x: a checkpoint of dy's rows is needed");
    if (!given && accumulate) refuse("accumulate: needs out");
    at::Tensor out = given ? *given : fresh({k.cols, dy.c}, at::kFloat, device);
    const Matrix o = matrix(out, "out", nullptr, dy.c);
    if (o.type != EF_TYPE_F32 || o.n != k.cols || out.device() != device)
        refuse("out: a float32 matrix of x's columns by dy's columns is needed");
    size_t bytes = 0;
    check(lib.checkpoint_weight_grad_workspace_bytes(dy.type, dy.n, k.cols, dy.c, dy.p(), dy.ld, &bytes),
          "ef_checkpoint_weight_grad_workspace_bytes");
    at::Tensor work;
    if (bytes) work = fresh({(int64_t)bytes}, at::kByte, device);
    const On on(device);
    check(lib.checkpoint_weight_grad(dy.type, dy.n, k.cols, dy.c, k.codes, k.scales, dy.p(), dy.ld, (float*)o.p(), o.ld,
                                     accumulate, bytes ? work.data_ptr() : nullptr, bytes, on.stream), "ef_checkpoint_weight_grad");
    if (given) {
        written(out);
        Py_INCREF(a[5]);
        return a[5];
    }
    return wrapped(std::move(out));
}

PyObject* token_logprob(PyObject* const* a) {            // logits, targets, temperature -> logp
    const Matrix x = matrix(a[0], "logits");
    const int64_t* const t = (const int64_t*)vec(a[1], x.n, "targets", x, at::kLong);
    const float temperature = (float)number(a[2]);
    at::Tensor logp = fresh({x.n}, at::kFloat, x.t.device());
    const On on(x.t.device());
    check(lib.token_logprob(x.type, x.n, x.c, x.p(), x.ld, t, temperature, (float*)logp.data_ptr(), on.stream), "ef_token_logprob");
    return wrapped(std::move(logp));
}

// logits, targets, old, adv, weights, ref, lo, hi, beta, temperature, need_grad, in_place -> loss, logp, token, grad
PyObject* policy_loss(PyObject* const* a) {
    const Matrix x = matrix(a[0], "logits");
    const int64_t* const t = (const int64_t*)vec(a[1], x.n, "targets", x, at::kLong);
    const float* const old = (const float*)vec(a[2], x.n, "old_logp", x);
    const float* const adv = (const float*)vec(a[3], x.n, "advantages", x);
    const float* const w = (const float*)vec(a[4], x.n, "weights", x);
    const float* const ref = a[5] == Py_None ? nullptr : (const float*)vec(a[5], x.n, "ref_logp", x);
    const float lo = (float)number(a[6]), hi = (float)number(a[7]), beta = (float)number(a[8]), temperature = (float)number(a[9]);
    const bool need_grad = truth(a[10]), in_place = truth(a[11]);
    const c10::Device device = x.t.device();
    if (need_grad && in_place) check_overwritable(x.t, "logits");
    at::Tensor grad;
    if (need_grad) grad = in_place ? x.t : fresh({x.n, x.c}, x.t.scalar_type(), device);
    at::Tensor loss = fresh({}, at::kFloat, device), logp = fresh({x.n}, at::kFloat, device), token = fresh({x.n}, at::kFloat, device);
    const On on(device);
    check(lib.policy_loss(x.type, x.n, x.c, x.p(), x.ld, t, old, adv, w, ref, lo, hi, beta, temperature, (float*)loss.data_ptr(),
                          (float*)logp.data_ptr(), (float*)token.data_ptr(), need_grad ? grad.data_ptr() : nullptr,
                          in_place ? x.ld : x.c, on.stream), "ef_policy_loss");
    if (need_grad && in_place) written(x.t);
    return pack(std::move(loss), std::move(logp), std::move(token), std::move(grad));
}

// bind(addresses in the order of the structure above, function that makes an exception of (status, name))
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr Py_ssize_t kCalls = sizeof(lib) / sizeof(void*);
    if (n != 2 || !PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != kCalls) {
        PyErr_SetString(PyExc_TypeError, "bind: a tuple of addresses and a function are needed");
        return nullptr;
    }
    void* at[kCalls];
    for (Py_ssize_t i = 0; i < kCalls; ++i) {
        at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], i));
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&lib, at, sizeof(lib));
    Py_XDECREF(status_error);
    Py_INCREF(a[1]);
    status_error = a[1];
    Py_RETURN_NONE;
}

// A call with a fixed number of positional arguments; C++ exceptions become Python's.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N || !status_error) {
        PyErr_SetString(PyExc_TypeError, status_error ? "wrong number of arguments" : "bind() comes first");
        return nullptr;
    }
    try {
        return F(a);
    } catch (const Refused&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}
#define EF_ENTRY(f, n) {#f, (PyCFunction)(void (*)(void))entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    EF_ENTRY(checkpoint_save, 1), EF_ENTRY(checkpoint_load, 5), EF_ENTRY(rmsnorm_forward, 5), EF_ENTRY(rmsnorm_backward, 9),
    EF_ENTRY(activation_forward, 4), EF_ENTRY(activation_backward, 6), EF_ENTRY(checkpoint_weight_grad, 7),
    EF_ENTRY(token_logprob, 3), EF_ENTRY(policy_loss, 12), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ef_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ef_torch() {
    PyObject* const m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", EF_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
