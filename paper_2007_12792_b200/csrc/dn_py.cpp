// Native marshalling of the Python entry points that a training loop calls per step: reads the fields of a Problem / Burgers
// object and the tensors' pointers, checks what the ctypes binding checks, calls the C entry point on the current stream.
// A call it does not recognise as plain (wrong type, device or layout of a tensor, a stream given) answers None, and the
// ctypes binding takes it, with its errors.  Also the two losses as autograd functions.
//
// The recurrence, the activations and the 8-bit tensors are marshalled here alone: their functions raise what is wrong with a tensor
// and answer the status.
//
// Why: marshalling through ctypes cost more than the launches of a small problem (64^2 x 8: 17.5 us per call, of which 7.5 us
// are the three launches), and the autograd function in Python 20 us more per direction.
#include <torch/extension.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Dtype.h>
#include <c10/core/AutogradState.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include "dn.h"

namespace {

struct Names {
    PyObject *dim, *nx, *ny, *nz, *batch, *nu_mode, *nu, *kl_modes, *kl_w, *f_const, *f, *bc_x0, *bc_x1, *flags, *bc_x0_b, *bc_x1_b, *nt, *T, *lam, *c,
        *rows, *cols, *dtype, *mix, *lengths, *format;
} N;

struct NotPlain {};                                     // thrown where the ctypes binding has to look

struct Attr {                                           // an attribute of a Python object, owned
    PyObject* o;
    Attr(PyObject* from, PyObject* name) : o(PyObject_GetAttr(from, name)) { if (!o) { PyErr_Clear(); throw NotPlain{}; } }
    ~Attr() { Py_DECREF(o); }
    Attr(const Attr&) = delete;
    int32_t i32() const {
        const long v = PyLong_AsLong(o);
        if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); throw NotPlain{}; }
        if (v < INT32_MIN || v > INT32_MAX) throw NotPlain{};
        return (int32_t)v;
    }
    float f32() const {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw NotPlain{}; }
        return (float)v;
    }
};

float* floats(PyObject* o) {                            // a contiguous float32 CUDA tensor, or None
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw NotPlain{};
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.scalar_type() != at::kFloat || !t.is_cuda() || !t.is_contiguous()) throw NotPlain{};
    return static_cast<float*>(t.data_ptr());
}
const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) throw NotPlain{};
    return THPVariable_Unpack(o);
}
const float* floats_of(PyObject* from, PyObject* name) { return floats(Attr(from, name).o); }      // the object keeps it alive

dn_problem problem_of(PyObject* o) {
    dn_problem p{};
    p.grid.dim = Attr(o, N.dim).i32(); p.grid.nx = Attr(o, N.nx).i32(); p.grid.ny = Attr(o, N.ny).i32();
    p.grid.nz = p.grid.dim == 3 ? Attr(o, N.nz).i32() : 1;
    p.batch = Attr(o, N.batch).i32(); p.nu_mode = Attr(o, N.nu_mode).i32(); p.kl_modes = Attr(o, N.kl_modes).i32();
    p.nu = floats_of(o, N.nu); p.kl_w = floats_of(o, N.kl_w); p.f = floats_of(o, N.f);
    p.f_const = Attr(o, N.f_const).f32(); p.bc_x0 = Attr(o, N.bc_x0).f32(); p.bc_x1 = Attr(o, N.bc_x1).f32();
    p.flags = (uint32_t)Attr(o, N.flags).i32();
    p.bc_x0_b = floats_of(o, N.bc_x0_b); p.bc_x1_b = floats_of(o, N.bc_x1_b);
    return p;
}
dn_burgers burgers_of(PyObject* o) {
    dn_burgers p{};
    p.nx = Attr(o, N.nx).i32(); p.nt = Attr(o, N.nt).i32(); p.batch = Attr(o, N.batch).i32();
    p.T = Attr(o, N.T).f32(); p.lambda = Attr(o, N.lam).f32(); p.flags = (uint32_t)Attr(o, N.flags).i32();
    p.c = floats_of(o, N.c);
    return p;
}
void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// C++ exceptions become Python ones by torch's own translation: an allocation that fails is a torch.OutOfMemoryError, what a
// Python callback (a saved-tensor hook) raised keeps its type and traceback.
template <class F>
PyObject* call(F f) {                                   // the status as an int, or None
    HANDLE_TH_ERRORS
    try {
        return PyLong_FromLong((long)f());
    } catch (const NotPlain&) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}
#define DN_NO_GIL(x) [&]() { dn_status s_; Py_BEGIN_ALLOW_THREADS s_ = (x); Py_END_ALLOW_THREADS return s_; }()
#define DN_ARGS(n) do { if (nargs != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; } } while (0)

PyObject* energy_grad(PyObject*, PyObject* const* a, Py_ssize_t nargs) {       // problem, u, gJ, J, r, workspace
    DN_ARGS(6);
    return call([&]() {
        const dn_problem p = problem_of(a[0]);
        const float *u = floats(a[1]), *gJ = floats(a[2]);
        float *J = floats(a[3]), *r = floats(a[4]);
        const at::Tensor& ws = tensor(a[5]);
        void *w = ws.data_ptr(), *s = current_stream();
        const size_t n = (size_t)ws.numel();
        return DN_NO_GIL(dn_energy_grad(&p, u, gJ, J, r, w, n, s));
    });
}
PyObject* energy(PyObject*, PyObject* const* a, Py_ssize_t nargs) {            // problem, u, J, workspace
    DN_ARGS(4);
    return call([&]() {
        const dn_problem p = problem_of(a[0]);
        const float* u = floats(a[1]);
        float* J = floats(a[2]);
        const at::Tensor& ws = tensor(a[3]);
        void *w = ws.data_ptr(), *s = current_stream();
        const size_t n = (size_t)ws.numel();
        return DN_NO_GIL(dn_energy(&p, u, J, w, n, s));
    });
}
PyObject* burgers_loss_grad(PyObject*, PyObject* const* a, Py_ssize_t nargs) { // problem, u, gL, L, parts, g, workspace
    DN_ARGS(7);
    return call([&]() {
        const dn_burgers p = burgers_of(a[0]);
        const float *u = floats(a[1]), *gL = floats(a[2]);
        float *L = floats(a[3]), *parts = floats(a[4]), *g = floats(a[5]);
        const at::Tensor& ws = tensor(a[6]);
        void *w = ws.data_ptr(), *s = current_stream();
        const size_t n = (size_t)ws.numel();
        return DN_NO_GIL(dn_burgers_loss_grad(&p, u, gL, L, parts, g, w, n, s, nullptr, nullptr));
    });
}

// ---- the losses as autograd functions: forward computes the loss and its gradient in one pass, backward scales it -----
struct LossFn : torch::autograd::Function<LossFn> {
    // status: out; p, q: the statement of the problem, one of them null (only read during forward)
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& u_in, int64_t batch, int64_t p, int64_t q, int64_t ws, int64_t ws_bytes,
                              int64_t status) {
        const at::Tensor u = u_in.contiguous();
        at::Tensor loss = at::empty({batch}, u.options()), g = at::empty_like(u);
        void* s = current_stream();
        dn_status* st = reinterpret_cast<dn_status*>(status);
        const float* up = static_cast<const float*>(u.data_ptr());
        float *lp = static_cast<float*>(loss.data_ptr()), *gp = static_cast<float*>(g.data_ptr());
        void* w = reinterpret_cast<void*>(ws);
        if (p) *st = dn_energy_grad(reinterpret_cast<const dn_problem*>(p), up, nullptr, lp, gp, w, (size_t)ws_bytes, s);
        else *st = dn_burgers_loss_grad(reinterpret_cast<const dn_burgers*>(q), up, nullptr, lp, nullptr, gp, w, (size_t)ws_bytes, s, nullptr, nullptr);
        ctx->save_for_backward({g});
        return loss;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const at::Tensor g = ctx->get_saved_variables()[0];
        std::vector<int64_t> shape((size_t)g.dim(), 1);
        shape[0] = -1;
        at::Tensor none;
        return {grads[0].reshape(shape).to(g.scalar_type()) * g, none, none, none, none, none, none};
    }
};

template <class P>
PyObject* loss(PyObject* const* a, const P& p, int64_t batch, bool fem) {      // u, problem, workspace
    const at::Tensor& u = tensor(a[0]);
    if (u.scalar_type() != at::kFloat || !u.is_cuda() || u.dim() < 1) throw NotPlain{};
    const at::Tensor& ws = tensor(a[2]);
    dn_status st = DN_OK;
    const int64_t pp = reinterpret_cast<int64_t>(&p);
    at::Tensor out;
    {
        pybind11::gil_scoped_release no_gil;
        out = LossFn::apply(u, batch, fem ? pp : (int64_t)0, fem ? (int64_t)0 : pp, reinterpret_cast<int64_t>(ws.data_ptr()), ws.numel(),
                            reinterpret_cast<int64_t>(&st));
    }
    if (st != DN_OK) return PyLong_FromLong((long)st);
    return THPVariable_Wrap(out);
}
template <class F>
PyObject* call_loss(F f) {                              // the loss, a status as an int, or None
    HANDLE_TH_ERRORS
    try {
        return f();
    } catch (const NotPlain&) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}
PyObject* energy_loss(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    DN_ARGS(3);
    return call_loss([&]() { const dn_problem p = problem_of(a[1]); return loss(a, p, p.batch, true); });
}
PyObject* burgers_loss(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    DN_ARGS(3);
    return call_loss([&]() { const dn_burgers p = burgers_of(a[1]); return loss(a, p, p.batch, false); });
}

// ---- the gated recurrence, activations, tensors in 8 bits ----------------------------------------------------------------
// Tensors of one call: all on one device, which is made the current one for the launch.
struct Device {
    c10::optional<c10::Device> one;
    void see(const at::Tensor& t, const char* name) {
        TORCH_CHECK_VALUE(t.is_cuda() && t.layout() == at::kStrided, name, ": expected a dense CUDA tensor (there is no CPU path)");
        TORCH_CHECK_VALUE(!t.is_neg(), name, ": a negated view of other numbers; pass its resolve_neg()");
        if (!one) one = t.device();
        TORCH_CHECK_VALUE(*one == t.device(), name, ": on ", t.device(), ", the tensors ahead of it on ", *one);
    }
};
const at::Tensor& a_tensor(PyObject* o, const char* name) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, ": expected a torch.Tensor");
    return THPVariable_Unpack(o);
}
const at::Tensor none_tensor;
const at::Tensor& maybe_tensor(PyObject* o, const char* name) { return o == Py_None ? none_tensor : a_tensor(o, name); }

int32_t type_code(at::ScalarType t, const char* name) {
    switch (t) {
        case at::kFloat: return DN_F32;
        case at::kBFloat16: return DN_BF16;
        case at::kHalf: return DN_F16;
        default: TORCH_CHECK_VALUE(false, name, ": expected float32, bfloat16 or float16, found ", t);
    }
}
at::ScalarType scalar_of(int32_t type) { return type == DN_F32 ? at::kFloat : type == DN_BF16 ? at::kBFloat16 : at::kHalf; }

bool adjacent(const at::Tensor& t) { return t.size(2) == 1 || t.stride(2) == 1; }

dn_rows rows_of(const at::Tensor& t, const char* name, const dn_scan& s, Device& d) {
    if (!t.defined()) return dn_rows{nullptr, 0, 0};
    d.see(t, name);
    TORCH_CHECK_VALUE(t.scalar_type() == scalar_of(s.type), name, ": expected ", scalar_of(s.type), ", found ", t.scalar_type());
    TORCH_CHECK_VALUE(t.dim() == 3 && t.size(0) == s.batch && t.size(1) == s.rows && t.size(2) == s.cols, name, ": expected shape [", s.batch, ", ", s.rows, ", ",
                      s.cols, "], found ", t.sizes());
    TORCH_CHECK_VALUE(t.numel() == 0 || adjacent(t), name, ": expected adjacent columns (a last stride of 1)");
    return dn_rows{t.data_ptr(), s.batch > 1 ? t.stride(0) : 0, s.rows > 1 ? t.stride(1) : 0};
}
float* edge_of(const at::Tensor& t, const char* name, const dn_scan& s, Device& d) {
    if (!t.defined()) return nullptr;
    d.see(t, name);
    TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat && t.is_contiguous() && t.dim() == 2 && t.size(0) == s.batch && t.size(1) == s.cols, name,
                      ": expected a contiguous float32 tensor [", s.batch, ", ", s.cols, "]");
    return static_cast<float*>(t.data_ptr());
}
const int32_t* lengths_of(const at::Tensor& t, const dn_scan& s, Device& d) {
    if (!t.defined()) return nullptr;
    d.see(t, "lengths");
    TORCH_CHECK_VALUE(t.scalar_type() == at::kInt && t.is_contiguous() && t.dim() == 1 && t.size(0) == s.batch, "lengths: expected a contiguous int32 tensor [",
                      s.batch, "]");
    return static_cast<const int32_t*>(t.data_ptr());
}
void bytes_checked(const at::Tensor& t, const char* name, Device& d) {
    d.see(t, name);
    TORCH_CHECK_VALUE(t.scalar_type() == at::kByte && t.is_contiguous(), name, ": expected a contiguous uint8 tensor");
}
int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
int32_t small_integer(PyObject* o, const char* name) {
    const int64_t v = integer(o);
    TORCH_CHECK_VALUE(v >= INT32_MIN && v <= INT32_MAX, name, ": ", v, " is out of range");
    return (int32_t)v;
}
struct Field {                                          // an attribute of a Scan, owned
    PyObject* o;
    Field(PyObject* from, PyObject* name) : o(PyObject_GetAttr(from, name)) { if (!o) throw python_error(); }
    ~Field() { Py_DECREF(o); }
    Field(const Field&) = delete;
};
dn_scan scan_of(PyObject* o, at::Tensor& lengths) {
    dn_scan s{};
    s.batch = small_integer(Field(o, N.batch).o, "batch");
    s.rows = small_integer(Field(o, N.rows).o, "rows");
    s.cols = small_integer(Field(o, N.cols).o, "cols");
    Field dtype(o, N.dtype), mix(o, N.mix), len(o, N.lengths);
    TORCH_CHECK_TYPE(THPDtype_Check(dtype.o), "dtype: expected a torch.dtype");
    s.type = type_code(reinterpret_cast<THPDtype*>(dtype.o)->scalar_type, "dtype");
    const int m = PyObject_IsTrue(mix.o);
    if (m < 0) throw python_error();
    s.flags = m ? DN_SCAN_MIX : 0u;
    s.format = small_integer(Field(o, N.format).o, "format");
    lengths = maybe_tensor(len.o, "lengths");
    return s;
}
void* stream_of(PyObject* o, const Device& d) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream(d.one->index()).stream();
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw python_error();
    return reinterpret_cast<void*>(v);
}
template <class F> PyObject* status(F f) {
    HANDLE_TH_ERRORS
    return PyLong_FromLong((long)f());
    END_HANDLE_TH_ERRORS
}

PyObject* scan_checkpoint_bytes(PyObject*, PyObject* const* a, Py_ssize_t nargs) {       // problem
    DN_ARGS(1);
    HANDLE_TH_ERRORS
    at::Tensor lengths;
    const dn_scan s = scan_of(a[0], lengths);
    return PyLong_FromSize_t(dn_scan_checkpoint_bytes(&s));
    END_HANDLE_TH_ERRORS
}
PyObject* scan_forward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {      // problem, g, x, h0, h, h_last, checkpoint, stream
    DN_ARGS(8);
    return status([&]() {
        at::Tensor lengths;
        dn_scan s = scan_of(a[0], lengths);
        Device d;
        const dn_rows g = rows_of(a_tensor(a[1], "g"), "g", s, d), x = rows_of(a_tensor(a[2], "x"), "x", s, d);
        const float* h0 = edge_of(maybe_tensor(a[3], "h0"), "h0", s, d);
        const dn_rows h = rows_of(a_tensor(a[4], "h"), "h", s, d);
        float* last = edge_of(maybe_tensor(a[5], "h_last"), "h_last", s, d);
        s.lengths = lengths_of(lengths, s, d);
        const at::Tensor& ck = maybe_tensor(a[6], "checkpoint");
        if (ck.defined()) bytes_checked(ck, "checkpoint", d);
        void *c = ck.defined() ? ck.data_ptr() : nullptr, *st = stream_of(a[7], d);
        const size_t n = ck.defined() ? (size_t)ck.numel() : 0;
        c10::cuda::CUDAGuard guard(*d.one);
        return DN_NO_GIL(dn_scan_forward(&s, &g, &x, h0, &h, last, c, n, st));
    });
}
PyObject* scan_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {     // problem, g, x, checkpoint, dh, dh_last, dg, dx, dh0, stream
    DN_ARGS(10);
    return status([&]() {
        at::Tensor lengths;
        dn_scan s = scan_of(a[0], lengths);
        Device d;
        const bool full = s.format == DN_SAVE_FULL;
        const dn_rows g = rows_of(full ? a_tensor(a[1], "g") : none_tensor, "g", s, d), x = rows_of(full ? a_tensor(a[2], "x") : none_tensor, "x", s, d);
        const at::Tensor& ck = a_tensor(a[3], "checkpoint");
        bytes_checked(ck, "checkpoint", d);
        const dn_rows dh = rows_of(maybe_tensor(a[4], "dh"), "dh", s, d);
        const float* dlast = edge_of(maybe_tensor(a[5], "dh_last"), "dh_last", s, d);
        const dn_rows dg = rows_of(a_tensor(a[6], "dg"), "dg", s, d), dx = rows_of(a_tensor(a[7], "dx"), "dx", s, d);
        float* dh0 = edge_of(maybe_tensor(a[8], "dh0"), "dh0", s, d);
        s.lengths = lengths_of(lengths, s, d);
        void *c = ck.data_ptr(), *st = stream_of(a[9], d);
        const size_t n = (size_t)ck.numel();
        c10::cuda::CUDAGuard guard(*d.one);
        return DN_NO_GIL(dn_scan_backward(&s, &g, &x, c, n, dh.data ? &dh : nullptr, dlast, &dg, &dx, dh0, st));
    });
}

at::Tensor new_bytes(size_t n, const at::Tensor& like) { return at::empty({(int64_t)(n ? n : 1)}, like.options().dtype(at::kByte)); }
at::Tensor with_adjacent_columns(const at::Tensor& u) {
    const at::Tensor t = u.defined() ? u.resolve_neg() : u;
    return !t.defined() || (t.dim() == 3 && (t.numel() == 0 || adjacent(t))) ? t : t.contiguous();
}
at::Tensor dense(const at::Tensor& t) { return t.defined() ? t.resolve_neg().contiguous() : t; }

dn_scan scan_like(const at::Tensor& g, bool mix, int64_t format) {
    TORCH_CHECK_VALUE(g.dim() == 3, "gate: expected shape [batch, rows, cols], found ", g.sizes());
    for (int k = 0; k < 3; ++k) TORCH_CHECK_VALUE(g.size(k) <= INT32_MAX, "gate: ", g.sizes(), " is out of range");
    dn_scan s{};
    s.batch = (int32_t)g.size(0); s.rows = (int32_t)g.size(1); s.cols = (int32_t)g.size(2);
    s.type = type_code(g.scalar_type(), "gate");
    s.flags = mix ? DN_SCAN_MIX : 0u;
    s.format = (int32_t)format;
    return s;
}
[[noreturn]] void refuse(dn_status st, const char* where) { TORCH_CHECK(false, where, ": ", dn_status_string(st), " (status ", (int)st, ")"); }

struct ScanFn : torch::autograd::Function<ScanFn> {
    static torch::autograd::variable_list run(const at::Tensor& g, const at::Tensor& x, const at::Tensor& h0, const at::Tensor& lengths, bool mix, int64_t format,
                                              bool keep, at::Tensor* checkpoint, dn_status* st) {
        dn_scan s = scan_like(g, mix, format);
        Device d;
        const dn_rows rg = rows_of(g, "gate", s, d), rx = rows_of(x, "x", s, d);
        const float* p0 = edge_of(h0, "h0", s, d);
        s.lengths = lengths_of(lengths, s, d);
        c10::cuda::CUDAGuard guard(*d.one);
        at::Tensor h = at::empty({s.batch, s.rows, s.cols}, g.options()), last = at::empty({s.batch, s.cols}, g.options().dtype(at::kFloat));
        if (keep) *checkpoint = new_bytes(dn_scan_checkpoint_bytes(&s), g);
        const dn_rows rh = rows_of(h, "h", s, d);
        *st = dn_scan_forward(&s, &rg, &rx, p0, &rh, static_cast<float*>(last.data_ptr()), keep ? checkpoint->data_ptr() : nullptr,
                              keep ? (size_t)checkpoint->numel() : 0, c10::cuda::getCurrentCUDAStream(d.one->index()).stream());
        return {h, last};
    }
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& g_in, const at::Tensor& x_in, c10::optional<at::Tensor> h0_in,
                                                  c10::optional<at::Tensor> lengths_in, bool mix, int64_t format, int64_t status) {
        const at::Tensor none, g = with_adjacent_columns(g_in), x = with_adjacent_columns(x_in);
        const at::Tensor h0 = h0_in ? dense(*h0_in) : none, lengths = lengths_in ? *lengths_in : none;
        at::Tensor checkpoint;
        auto out = run(g, x, h0, lengths, mix, format, true, &checkpoint, reinterpret_cast<dn_status*>(status));
        // uint8: what packs the saved tensors of a step into 8 bits leaves the states in 32
        torch::autograd::variable_list keep{checkpoint};
        if (format == DN_SAVE_FULL) { keep.push_back(g); keep.push_back(x); }
        if (lengths.defined()) keep.push_back(lengths);                // last
        ctx->save_for_backward(std::move(keep));
        ctx->set_materialize_grads(false);
        ctx->saved_data["mix"] = mix;
        ctx->saved_data["h0"] = h0.defined();
        ctx->saved_data["format"] = format;
        ctx->saved_data["shape"] = out[0].sizes();
        ctx->saved_data["type"] = (int64_t)type_code(g.scalar_type(), "gate");
        return out;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "gated_scan: the gradients are not differentiable again (create_graph)");
        const at::Tensor none;
        if (!grads[0].defined() && !grads[1].defined()) return {none, none, none, none, none, none, none};
        const auto saved = ctx->get_saved_variables();
        const auto shape = ctx->saved_data["shape"].toIntVector();
        dn_scan s{};
        s.batch = (int32_t)shape[0]; s.rows = (int32_t)shape[1]; s.cols = (int32_t)shape[2];
        s.type = (int32_t)ctx->saved_data["type"].toInt();
        s.flags = ctx->saved_data["mix"].toBool() ? DN_SCAN_MIX : 0u;
        s.format = (int32_t)ctx->saved_data["format"].toInt();
        const bool full = s.format == DN_SAVE_FULL;
        const at::Tensor &ck = saved[0], dh = with_adjacent_columns(grads[0]), dlast = dense(grads[1]);
        const at::Tensor g = full ? with_adjacent_columns(saved[1]) : none, x = full ? with_adjacent_columns(saved[2]) : none;
        Device d;
        bytes_checked(ck, "checkpoint", d);
        c10::cuda::CUDAGuard guard(*d.one);
        const auto fields = ck.options().dtype(scalar_of(s.type));
        at::Tensor dg = at::empty(shape, fields), dx = at::empty(shape, fields), dh0;
        if (ctx->saved_data["h0"].toBool() && ctx->needs_input_grad(2)) dh0 = at::empty({s.batch, s.cols}, ck.options().dtype(at::kFloat));
        const dn_rows rg = rows_of(g, "gate", s, d), rx = rows_of(x, "x", s, d), rd = rows_of(dh, "dh", s, d), rdg = rows_of(dg, "dg", s, d), rdx = rows_of(dx, "dx", s, d);
        const float* pl = edge_of(dlast, "dh_last", s, d);
        s.lengths = lengths_of(saved.size() > (full ? 3u : 1u) ? saved.back() : none, s, d);
        const dn_status st = dn_scan_backward(&s, &rg, &rx, ck.data_ptr(), (size_t)ck.numel(), rd.data ? &rd : nullptr, pl, &rdg, &rdx,
                                              dh0.defined() ? static_cast<float*>(dh0.data_ptr()) : nullptr,
                                              c10::cuda::getCurrentCUDAStream(d.one->index()).stream());
        if (st != DN_OK) refuse(st, "dn_scan_backward");
        return {dg, dx, dh0, none, none, none, none};
    }
};

// A tensor with a tangent asks for no gradient: without this it would pass for one that nothing is to be derived from, and the
// result's missing tangent for zero.
void no_tangents(std::initializer_list<at::Tensor> ts, const char* where) {
    if (!c10::AutogradState::get_tls_state().get_fw_grad_mode()) return;
    for (const at::Tensor& t : ts)
        TORCH_CHECK_NOT_IMPLEMENTED(!t.defined() || !t._fw_grad(0).defined(), where, ": no forward-mode derivatives (torch.autograd.forward_ad)");
}
bool wants_grad(std::initializer_list<at::Tensor> ts) {
    if (!at::GradMode::is_enabled()) return false;
    for (const at::Tensor& t : ts)
        if (t.defined() && t.requires_grad()) return true;
    return false;
}

PyObject* gated_scan(PyObject*, PyObject* const* a, Py_ssize_t nargs) {        // gate, x, h0, lengths, mix, format: (h, h_last), or a status
    DN_ARGS(6);
    HANDLE_TH_ERRORS
    const at::Tensor &g = a_tensor(a[0], "gate"), &x = a_tensor(a[1], "x"), &h0 = maybe_tensor(a[2], "h0"), &lengths = maybe_tensor(a[3], "lengths");
    const int mix = PyObject_IsTrue(a[4]);
    if (mix < 0) throw python_error();
    const int64_t format = integer(a[5]);
    no_tangents({g, x, h0}, "gated_scan");
    dn_status st = DN_OK;
    torch::autograd::variable_list out;
    {
        pybind11::gil_scoped_release no_gil;
        if (wants_grad({g, x, h0})) {                   // (an undefined tensor may not be an argument of an autograd function)
            using Maybe = c10::optional<at::Tensor>;
            out = ScanFn::apply(g, x, h0.defined() ? Maybe(h0) : Maybe(), lengths.defined() ? Maybe(lengths) : Maybe(), mix != 0, format, reinterpret_cast<int64_t>(&st));
        }
        else out = ScanFn::run(with_adjacent_columns(g), with_adjacent_columns(x), dense(h0), lengths, mix != 0, format, false, nullptr, &st);
    }
    if (st != DN_OK) return PyLong_FromLong((long)st);
    PyObject* r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(out[0]));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(out[1]));
    return r;
    END_HANDLE_TH_ERRORS
}

struct ActivationFn : torch::autograd::Function<ActivationFn> {
    static at::Tensor run(const at::Tensor& x, int64_t kind, int64_t format, bool keep, at::Tensor* packed, dn_status* st) {
        const int32_t type = type_code(x.scalar_type(), "x");
        Device d;
        d.see(x, "x");
        c10::cuda::CUDAGuard guard(*d.one);
        at::Tensor y = at::empty_like(x);
        if (keep) *packed = new_bytes(dn_packed_bytes(x.numel()), x);
        if (x.numel() > 0)
            *st = dn_activation_forward(x.numel(), type, (int32_t)kind, x.data_ptr(), y.data_ptr(), (int32_t)format, keep ? packed->data_ptr() : nullptr,
                                        c10::cuda::getCurrentCUDAStream(d.one->index()).stream());
        return y;
    }
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, int64_t kind, int64_t format, int64_t status) {
        at::Tensor packed;
        const at::Tensor y = run(dense(x), kind, format, true, &packed, reinterpret_cast<dn_status*>(status));
        ctx->save_for_backward({packed});
        ctx->set_materialize_grads(false);
        ctx->saved_data["kind"] = kind;
        ctx->saved_data["format"] = format;
        return y;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "activation: the gradient is not differentiable again (create_graph)");
        const at::Tensor none;
        if (!grads[0].defined()) return {none, none, none, none};
        const at::Tensor packed = ctx->get_saved_variables()[0], dy = dense(grads[0]);
        Device d;
        bytes_checked(packed, "the saved input", d);
        d.see(dy, "dy");
        c10::cuda::CUDAGuard guard(*d.one);
        at::Tensor dx = at::empty_like(dy);
        if (dy.numel() == 0) return {dx, none, none, none};
        const dn_status st = dn_activation_backward(dy.numel(), type_code(dy.scalar_type(), "dy"), (int32_t)ctx->saved_data["kind"].toInt(), packed.data_ptr(),
                                                    (int32_t)ctx->saved_data["format"].toInt(), dy.data_ptr(), dx.data_ptr(),
                                                    c10::cuda::getCurrentCUDAStream(d.one->index()).stream());
        if (st != DN_OK) refuse(st, "dn_activation_backward");
        return {dx, none, none, none};
    }
};

PyObject* activation(PyObject*, PyObject* const* a, Py_ssize_t nargs) {        // x, kind, format: y, or a status
    DN_ARGS(3);
    HANDLE_TH_ERRORS
    const at::Tensor& x = a_tensor(a[0], "x");
    const int64_t kind = integer(a[1]), format = integer(a[2]);
    no_tangents({x}, "activation");
    dn_status st = DN_OK;
    at::Tensor y;
    {
        pybind11::gil_scoped_release no_gil;
        if (wants_grad({x})) y = ActivationFn::apply(x, kind, format, reinterpret_cast<int64_t>(&st));
        else y = ActivationFn::run(dense(x), kind, format, false, nullptr, &st);
    }
    if (st != DN_OK) return PyLong_FromLong((long)st);
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// the caller's buffers: src / dst contiguous, packed uint8 of dn_packed_bytes(numel) or more
void flat_checked(const at::Tensor& t, const char* name, const at::Tensor& packed, int64_t n, Device& d) {
    d.see(t, name);
    TORCH_CHECK_VALUE(t.is_contiguous(), name, ": expected a contiguous tensor");
    if (!packed.defined()) return;
    bytes_checked(packed, "packed", d);
    TORCH_CHECK_VALUE((size_t)packed.numel() >= dn_packed_bytes(n), "packed: ", packed.numel(), " bytes, expected ", dn_packed_bytes(n));
}
PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t nargs) {              // src, format, packed, stream
    DN_ARGS(4);
    return status([&]() {
        const at::Tensor &t = a_tensor(a[0], "src"), &p = a_tensor(a[2], "packed");
        Device d;
        flat_checked(t, "src", p, t.numel(), d);
        const int32_t type = type_code(t.scalar_type(), "src"), format = small_integer(a[1], "format");
        void* st = stream_of(a[3], d);
        c10::cuda::CUDAGuard guard(*d.one);
        return DN_NO_GIL(dn_pack(t.numel(), type, t.data_ptr(), format, p.data_ptr(), st));
    });
}
PyObject* unpack(PyObject*, PyObject* const* a, Py_ssize_t nargs) {            // packed, format, dst, stream
    DN_ARGS(4);
    return status([&]() {
        const at::Tensor &p = a_tensor(a[0], "packed"), &t = a_tensor(a[2], "dst");
        Device d;
        flat_checked(t, "dst", p, t.numel(), d);
        const int32_t type = type_code(t.scalar_type(), "dst"), format = small_integer(a[1], "format");
        void* st = stream_of(a[3], d);
        c10::cuda::CUDAGuard guard(*d.one);
        return DN_NO_GIL(dn_unpack(t.numel(), type, p.data_ptr(), format, t.data_ptr(), st));
    });
}
PyObject* packed(PyObject*, PyObject* const* a, Py_ssize_t nargs) {            // src of any layout, format: the packed tensor, or a status
    DN_ARGS(2);
    HANDLE_TH_ERRORS
    const at::Tensor& src = a_tensor(a[0], "src");
    const int32_t type = type_code(src.scalar_type(), "src"), format = small_integer(a[1], "format");
    Device d;
    d.see(src.resolve_neg(), "src");
    c10::cuda::CUDAGuard guard(*d.one);
    at::Tensor out;
    dn_status st = DN_OK;
    {
        pybind11::gil_scoped_release no_gil;
        at::NoGradGuard no_grad;
        const at::Tensor t = dense(src);
        out = new_bytes(dn_packed_bytes(t.numel()), t);
        if (t.numel() > 0) st = dn_pack(t.numel(), type, t.data_ptr(), format, out.data_ptr(), c10::cuda::getCurrentCUDAStream(d.one->index()).stream());
    }
    if (st != DN_OK) return PyLong_FromLong((long)st);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}
PyObject* unpacked(PyObject*, PyObject* const* a, Py_ssize_t nargs) {          // packed, format, shape, dtype: a new tensor, or a status
    DN_ARGS(4);
    HANDLE_TH_ERRORS
    const at::Tensor& p = a_tensor(a[0], "packed");
    const int32_t format = small_integer(a[1], "format");
    TORCH_CHECK_TYPE(PyTuple_Check(a[2]) && THPDtype_Check(a[3]), "unpack: expected a shape and a dtype");
    std::vector<int64_t> shape;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[2]); ++i) shape.push_back(integer(PyTuple_GET_ITEM(a[2], i)));
    const at::ScalarType dtype = reinterpret_cast<THPDtype*>(a[3])->scalar_type;
    const int32_t type = type_code(dtype, "dtype");
    Device d;
    bytes_checked(p, "packed", d);
    c10::cuda::CUDAGuard guard(*d.one);
    at::Tensor out;
    dn_status st = DN_OK;
    {
        pybind11::gil_scoped_release no_gil;
        out = at::empty(shape, p.options().dtype(dtype));
        TORCH_CHECK_VALUE((size_t)p.numel() >= dn_packed_bytes(out.numel()), "packed: ", p.numel(), " bytes, expected ", dn_packed_bytes(out.numel()));
        if (out.numel() > 0) st = dn_unpack(out.numel(), type, p.data_ptr(), format, out.data_ptr(), c10::cuda::getCurrentCUDAStream(d.one->index()).stream());
    }
    if (st != DN_OK) return PyLong_FromLong((long)st);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}
PyObject* activation_forward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {          // kind, x, y, format, packed, stream
    DN_ARGS(6);
    return status([&]() {
        const at::Tensor &x = a_tensor(a[1], "x"), &y = a_tensor(a[2], "y"), &p = maybe_tensor(a[4], "packed");
        Device d;
        flat_checked(x, "x", p, x.numel(), d);
        flat_checked(y, "y", none_tensor, 0, d);
        TORCH_CHECK_VALUE(y.numel() == x.numel() && y.scalar_type() == x.scalar_type(), "y: expected the size and type of x");
        const int32_t type = type_code(x.scalar_type(), "x"), kind = small_integer(a[0], "kind"), format = small_integer(a[3], "format");
        void *st = stream_of(a[5], d), *q = p.defined() ? p.data_ptr() : nullptr;
        c10::cuda::CUDAGuard guard(*d.one);
        return DN_NO_GIL(dn_activation_forward(x.numel(), type, kind, x.data_ptr(), y.data_ptr(), format, q, st));
    });
}
PyObject* activation_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {         // kind, packed, format, dy, dx, stream
    DN_ARGS(6);
    return status([&]() {
        const at::Tensor &p = a_tensor(a[1], "packed"), &dy = a_tensor(a[3], "dy"), &dx = a_tensor(a[4], "dx");
        Device d;
        flat_checked(dy, "dy", p, dy.numel(), d);
        flat_checked(dx, "dx", none_tensor, 0, d);
        TORCH_CHECK_VALUE(dx.numel() == dy.numel() && dx.scalar_type() == dy.scalar_type(), "dx: expected the size and type of dy");
        const int32_t type = type_code(dy.scalar_type(), "dy"), kind = small_integer(a[0], "kind"), format = small_integer(a[2], "format");
        void* st = stream_of(a[5], d);
        c10::cuda::CUDAGuard guard(*d.one);
        return DN_NO_GIL(dn_activation_backward(dy.numel(), type, kind, p.data_ptr(), format, dy.data_ptr(), dx.data_ptr(), st));
    });
}

PyMethodDef methods[] = {
    {"scan_checkpoint_bytes", (PyCFunction)(void (*)(void))scan_checkpoint_bytes, METH_FASTCALL, nullptr},
    {"scan_forward", (PyCFunction)(void (*)(void))scan_forward, METH_FASTCALL, nullptr},
    {"scan_backward", (PyCFunction)(void (*)(void))scan_backward, METH_FASTCALL, nullptr},
    {"gated_scan", (PyCFunction)(void (*)(void))gated_scan, METH_FASTCALL, nullptr},
    {"activation", (PyCFunction)(void (*)(void))activation, METH_FASTCALL, nullptr},
    {"packed", (PyCFunction)(void (*)(void))packed, METH_FASTCALL, nullptr},
    {"unpacked", (PyCFunction)(void (*)(void))unpacked, METH_FASTCALL, nullptr},
    {"pack", (PyCFunction)(void (*)(void))pack, METH_FASTCALL, nullptr},
    {"unpack", (PyCFunction)(void (*)(void))unpack, METH_FASTCALL, nullptr},
    {"activation_forward", (PyCFunction)(void (*)(void))activation_forward, METH_FASTCALL, nullptr},
    {"activation_backward", (PyCFunction)(void (*)(void))activation_backward, METH_FASTCALL, nullptr},
    {"energy_grad", (PyCFunction)(void (*)(void))energy_grad, METH_FASTCALL, nullptr},
    {"energy", (PyCFunction)(void (*)(void))energy, METH_FASTCALL, nullptr},
    {"burgers_loss_grad", (PyCFunction)(void (*)(void))burgers_loss_grad, METH_FASTCALL, nullptr},
    {"energy_loss", (PyCFunction)(void (*)(void))energy_loss, METH_FASTCALL, nullptr},
    {"burgers_loss", (PyCFunction)(void (*)(void))burgers_loss, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
#define DN_NAME(x) N.x = PyUnicode_InternFromString(#x);
    DN_NAME(dim) DN_NAME(nx) DN_NAME(ny) DN_NAME(nz) DN_NAME(batch) DN_NAME(nu_mode) DN_NAME(nu) DN_NAME(kl_modes) DN_NAME(kl_w) DN_NAME(f_const)
    DN_NAME(f) DN_NAME(bc_x0) DN_NAME(bc_x1) DN_NAME(flags) DN_NAME(bc_x0_b) DN_NAME(bc_x1_b) DN_NAME(nt) DN_NAME(T) DN_NAME(lam) DN_NAME(c)
    DN_NAME(rows) DN_NAME(cols) DN_NAME(dtype) DN_NAME(mix) DN_NAME(lengths) DN_NAME(format)
#undef DN_NAME
    return PyModule_Create(&module);
}
