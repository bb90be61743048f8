// The binding's common calls without an interpreter in the way: a planned stack bound to torch tensors (module _bs_torch).
//
// One call of a small stack is a launch of a few microseconds; reading shapes, asking for memory and passing pointers through ctypes took
// three times that (Stack.run 10.3 us, run and backward 21 us, the module under autograd 85 to 95 us, whatever the kernels).  Here the same
// checks, allocations and calls are made natively for the plain case -- dense tensors of the plan's shape, type, memory order and device on
// the current stream -- and every method returns None for anything else, which the Python code then handles (or refuses) as it always does.
//
// The library is reached through the function addresses the Python side has loaded: this file links against torch only.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/PythonFallbackKernel.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <c10/util/SmallVector.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <array>
#include <cstdint>
#include <map>
#include <memory>
#include <mutex>
#include <utility>
#include <vector>

#include "brainslug.h"

namespace {

using Shape = std::array<int64_t, 4>;
using RunFn = int (*)(const void *, const void *, int64_t, const void *const *, void *, int64_t, int32_t *const *, void *, uint64_t, void *);
using BackwardFn = int (*)(const void *, const void *, int64_t, const void *const *, const int32_t *const *, const void *, int64_t, void *, int64_t,
                           void *const *, void *, uint64_t, void *);
using DestroyFn = void (*)(void *);

// A failed library call, raised in Python as the binding's own error (the binding sets the class).
PyObject *g_error = nullptr;
struct CallFailed : std::exception {
    int status;
    const char *where;
    CallFailed(int s, const char *w) : status(s), where(w) {}
    const char *what() const noexcept override { return where; }
};

PyObject *failed(const CallFailed &e)
{
    if (g_error) {
        PyObject *err = PyObject_CallFunction(g_error, "is", e.status, e.where);
        if (err) {
            PyErr_SetObject(reinterpret_cast<PyObject *>(Py_TYPE(err)), err);
            Py_DECREF(err);
        }
    } else {
        PyErr_SetString(PyExc_RuntimeError, e.where);
    }
    return nullptr;
}

// What a planned stack's handle needs beside it.  Shared between the Python object and the graph nodes recorded with it; the last one
// destroys the handle, unless it was closed before.
struct Plan {
    void *handle = nullptr;
    RunFn run = nullptr;
    BackwardFn backward = nullptr;
    DestroyFn destroy = nullptr;
    Shape in{}, out{};
    std::vector<Shape> res, idx;
    at::ScalarType dtype = at::kFloat;
    at::MemoryFormat mf = at::MemoryFormat::Contiguous;
    uint64_t ws_bytes = 0, bwd_ws_bytes = 0;
    bool bwd_planned = false, bwd_reads_picks = true;
    std::mutex mutex;
    // one workspace per (device, stream) and direction: runs on different streams may overlap
    using Buffers = std::map<std::pair<int, void *>, at::Tensor>;
    Buffers ws[2];

    ~Plan()
    {
        if (handle) destroy(handle);
    }
    // Closed or planned anew: the handle is the Python object's again, nothing runs here any more.
    void *release()
    {
        Buffers old[2];
        std::lock_guard<std::mutex> lock(mutex);
        void *h = handle;
        handle = nullptr;
        for (int i = 0; i < 2; ++i) old[i].swap(ws[i]);
        return h;
    }
    // Nothing is allocated or freed under the mutex: the allocator may call into the interpreter, whose lock the thread that waits for the
    // mutex may hold.
    at::Tensor workspace(bool bwd, const at::Device &dev, void *stream)
    {
        const uint64_t n = bwd ? bwd_ws_bytes : ws_bytes;
        if (!n) return {};
        const Buffers::key_type key{dev.index(), stream};
        {
            std::lock_guard<std::mutex> lock(mutex);
            const auto it = ws[bwd].find(key);
            if (it != ws[bwd].end()) return it->second;
        }
        const at::Tensor t = at::empty({(int64_t)n}, at::TensorOptions().dtype(at::kByte).device(dev));
        std::lock_guard<std::mutex> lock(mutex);
        return ws[bwd].emplace(key, t).first->second;  // (another thread's, if it was faster)
    }
    at::TensorOptions options(const at::Tensor &like) const { return at::TensorOptions().dtype(dtype).device(like.device()); }
};

// A dense tensor of this shape in the plan's memory order, on `dev`, whose memory can be addressed.
bool plain(const Plan &p, const at::Tensor &t, const Shape &shape, at::ScalarType dtype, const at::Device *dev)
{
    return t.defined() && t.is_cuda() && t.scalar_type() == dtype && t.dim() == 4 && t.sizes() == at::IntArrayRef(shape.data(), 4) && t.has_storage() &&
           (!dev || t.device() == *dev) && t.is_contiguous(p.mf);
}

// Elements between the images of a tensor that the library can read in place: dense (0), or a channel slice of a dense tensor whose
// images (channels-last: pixels) keep the alignment; -1: neither.
int64_t slice_stride(const Plan &p, const at::Tensor &t)
{
    if (reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 != 0) return -1;
    if (t.is_contiguous(p.mf)) return 0;
    const int64_t n = t.size(0), c = t.size(1), h = t.size(2), w = t.size(3), es = (int64_t)t.element_size();
    const int64_t sn = t.stride(0), sc = t.stride(1), sh = t.stride(2), sw = t.stride(3);
    if (p.mf == at::MemoryFormat::Contiguous) {
        const bool slice = (w == 1 || sw == 1) && (h == 1 || sh == w) && (c == 1 || sc == h * w) && (n == 1 || sn >= c * h * w);
        const int64_t stride = n > 1 ? sn : c * h * w;
        return slice && stride * es % 16 == 0 ? stride : -1;
    }
    const int64_t ct = w > 1 ? sw : h > 1 ? sh : n > 1 ? sn : c;  // channels of the larger tensor
    const bool slice = ct >= c && (c == 1 || sc == 1) && (w == 1 || sw == ct) && (h == 1 || sh == w * ct) && (n == 1 || sn == h * w * ct);
    return slice && ct * es % 16 == 0 ? h * w * ct : -1;
}

bool modes_active() { return c10::impl::dispatch_mode_enabled(); }

// out and (if wanted) picks for x; the launch.  The caller has checked the operands.
void run_forward(Plan &p, const at::Tensor &x, const std::vector<at::Tensor> &res, at::Tensor &out, std::vector<at::Tensor> &picks, bool want_picks = true)
{
    out = at::empty(at::IntArrayRef(p.out.data(), 4), p.options(x).memory_format(p.mf));
    picks.clear();
    if (want_picks)
        for (const Shape &s : p.idx) picks.push_back(at::empty(at::IntArrayRef(s.data(), 4), p.options(x).dtype(at::kInt).memory_format(p.mf)));
    void *stream = c10::hip::getCurrentHIPStream(x.device().index()).stream();
    const at::Tensor ws = p.workspace(false, x.device(), stream);
    c10::SmallVector<const void *, 4> rp;
    c10::SmallVector<int32_t *, 4> ip;
    for (const at::Tensor &r : res) rp.push_back(r.data_ptr());
    for (const at::Tensor &t : picks) ip.push_back(static_cast<int32_t *>(t.data_ptr()));
    const int rc = p.run(p.handle, x.data_ptr(), 0, res.empty() ? nullptr : rp.data(), out.data_ptr(), 0, picks.empty() ? nullptr : ip.data(),
                         ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? (uint64_t)ws.numel() : 0, stream);
    if (rc != 0) throw CallFailed(rc, "bs_stack_run");
}

// `need`: input, then residuals.
void run_backward(Plan &p, const at::Tensor &x, const std::vector<at::Tensor> &res, const at::Tensor &dy, int64_t dy_stride, const std::vector<at::Tensor> &picks,
                  const std::vector<bool> &need, at::Tensor &gx, std::vector<at::Tensor> &gres)
{
    if (need[0]) gx = at::empty(at::IntArrayRef(p.in.data(), 4), p.options(x).memory_format(p.mf));
    gres.assign(res.size(), at::Tensor());
    for (size_t i = 0; i < res.size(); ++i)
        if (need[i + 1]) gres[i] = at::empty(at::IntArrayRef(p.res[i].data(), 4), p.options(x).memory_format(p.mf));
    void *stream = c10::hip::getCurrentHIPStream(x.device().index()).stream();
    const at::Tensor ws = p.workspace(true, x.device(), stream);
    c10::SmallVector<const void *, 4> rp;
    c10::SmallVector<void *, 4> gp;
    c10::SmallVector<const int32_t *, 4> ip;
    for (size_t i = 0; i < res.size(); ++i) {
        rp.push_back(res[i].data_ptr());
        gp.push_back(gres[i].defined() ? gres[i].data_ptr() : nullptr);
    }
    for (const at::Tensor &t : picks) ip.push_back(t.defined() ? static_cast<const int32_t *>(t.data_ptr()) : nullptr);
    const int rc = p.backward(p.handle, x.data_ptr(), 0, res.empty() ? nullptr : rp.data(), picks.empty() ? nullptr : ip.data(), dy.data_ptr(), dy_stride,
                              gx.defined() ? gx.data_ptr() : nullptr, 0, res.empty() ? nullptr : gp.data(), ws.defined() ? ws.data_ptr() : nullptr,
                              ws.defined() ? (uint64_t)ws.numel() : 0, stream);
    if (rc != 0) throw CallFailed(rc, "bs_stack_backward");
}

// The stack as one node of the autograd graph: keeps its operands (through torch's saved variables) and the picks.
struct StackNode : torch::autograd::Function<StackNode> {
    struct Held : torch::CustomClassHolder {
        std::shared_ptr<Plan> plan;
        std::vector<at::Tensor> picks;
    };
    static at::Tensor forward(torch::autograd::AutogradContext *ctx, const std::shared_ptr<Plan> &plan, const at::Tensor &x, at::TensorList residuals)
    {
        auto held = c10::make_intrusive<Held>();
        held->plan = plan;
        const std::vector<at::Tensor> res = residuals.vec();
        at::Tensor out;
        {
            pybind11::gil_scoped_release no_gil;
            run_forward(*plan, x, res, out, held->picks, plan->bwd_reads_picks);
        }
        torch::autograd::variable_list saved{x};
        saved.insert(saved.end(), res.begin(), res.end());
        ctx->save_for_backward(std::move(saved));
        ctx->saved_data["held"] = c10::IValue::make_capsule(std::move(held));
        return out;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext *ctx, torch::autograd::variable_list grads)
    {
        const auto held = c10::static_intrusive_pointer_cast<Held>(ctx->saved_data["held"].toCapsule());
        Plan &p = *held->plan;
        const auto saved = ctx->get_saved_variables();
        const at::Tensor &x = saved[0];
        const std::vector<at::Tensor> res(saved.begin() + 1, saved.end());
        TORCH_CHECK(p.handle, "the stack of this graph was closed, or its parameters were read again, before the backward pass");
        std::vector<bool> need(1 + res.size());
        for (size_t i = 0; i < need.size(); ++i) need[i] = ctx->needs_input_grad(i);
        // the upstream gradient has the output's shape and type and is read in place when it is dense or a channel slice
        at::Tensor dy = grads[0];
        int64_t stride = slice_stride(p, dy);
        if (stride < 0) {
            dy = dy.contiguous(p.mf);
            stride = 0;
        }
        at::Tensor gx;
        std::vector<at::Tensor> gres;
        try {
            run_backward(p, x, res, dy, stride, held->picks, need, gx, gres);
        } catch (const CallFailed &e) {  // raised in Python as the binding's error
            pybind11::gil_scoped_acquire gil;
            failed(e);
            python_error err;
            err.persist();
            throw err;
        }
        torch::autograd::variable_list all{at::Tensor(), gx};  // (the plan has no gradient)
        all.insert(all.end(), gres.begin(), gres.end());
        return all;
    }
};

// ---------------------------------------------------------------------------------------------------- Python type
struct PlanObject {
    PyObject_HEAD
    std::shared_ptr<Plan> *plan;
};

bool read_shape(PyObject *o, Shape &s)
{
    PyObject *f = PySequence_Fast(o, "shape");
    if (!f) return false;
    const bool four = PySequence_Fast_GET_SIZE(f) == 4;
    if (!four) PyErr_SetString(PyExc_ValueError, "a shape has four dimensions");
    for (int i = 0; four && i < 4; ++i) s[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(f, i));
    Py_DECREF(f);
    return four && !PyErr_Occurred();
}
bool read_shapes(PyObject *o, std::vector<Shape> &v)
{
    PyObject *f = PySequence_Fast(o, "shapes");
    if (!f) return false;
    bool ok = true;
    for (Py_ssize_t i = 0; ok && i < PySequence_Fast_GET_SIZE(f); ++i) {
        Shape s;
        ok = read_shape(PySequence_Fast_GET_ITEM(f, i), s);
        if (ok) v.push_back(s);
    }
    Py_DECREF(f);
    return ok;
}

// Plan(addresses (run, backward, destroy), handle, in_shape, out_shape, dtype 0 / 1 / 2, channels_last, residual shapes, index shapes, workspace bytes)
PyObject *plan_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    HANDLE_TH_ERRORS
    unsigned long long run, backward, destroy, handle, ws;
    PyObject *in, *out, *res, *idx;
    int dtype, nhwc;
    if (!PyArg_ParseTuple(args, "(KKK)KOOipOOK", &run, &backward, &destroy, &handle, &in, &out, &dtype, &nhwc, &res, &idx, &ws)) return nullptr;
    auto p = std::make_shared<Plan>();
    p->run = reinterpret_cast<RunFn>(run);
    p->backward = reinterpret_cast<BackwardFn>(backward);
    p->destroy = reinterpret_cast<DestroyFn>(destroy);
    p->dtype = dtype == 0 ? at::kFloat : dtype == 1 ? at::kBFloat16 : at::kHalf;
    p->mf = nhwc ? at::MemoryFormat::ChannelsLast : at::MemoryFormat::Contiguous;
    p->ws_bytes = ws;
    if (!read_shape(in, p->in) || !read_shape(out, p->out) || !read_shapes(res, p->res) || !read_shapes(idx, p->idx)) return nullptr;
    PlanObject *self = reinterpret_cast<PlanObject *>(type->tp_alloc(type, 0));
    if (!self) return nullptr;
    p->handle = reinterpret_cast<void *>(handle);
    self->plan = new std::shared_ptr<Plan>(std::move(p));
    return reinterpret_cast<PyObject *>(self);
    END_HANDLE_TH_ERRORS
}

void plan_dealloc(PyObject *o)
{
    PlanObject *self = reinterpret_cast<PlanObject *>(o);
    delete self->plan;
    PyTypeObject *type = Py_TYPE(o);
    type->tp_free(o);
    Py_DECREF(type);
}

Plan &plan_of(PyObject *o) { return **reinterpret_cast<PlanObject *>(o)->plan; }

const at::Tensor *tensor_of(PyObject *o)
{
    return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr;  // (subclasses: Python)
}

// x and a tuple or list of residuals, checked; false: not the plain case (no error set)
bool operands(Plan &p, PyObject *xo, PyObject *ro, const at::Tensor *&x, std::vector<at::Tensor> &res)
{
    x = tensor_of(xo);
    if (!p.handle || !x || modes_active() || !plain(p, *x, p.in, p.dtype, nullptr)) return false;
    if (!PyTuple_Check(ro) && !PyList_Check(ro)) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(ro);
    if ((size_t)n != p.res.size()) return false;
    const at::Device dev = x->device();
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor *r = tensor_of(PySequence_Fast_GET_ITEM(ro, i));
        if (!r || !plain(p, *r, p.res[i], p.dtype, &dev)) return false;
        res.push_back(*r);
    }
    return true;
}

PyObject *wrap_list(std::vector<at::Tensor> &v)
{
    PyObject *l = PyList_New((Py_ssize_t)v.size());
    if (!l) return nullptr;
    for (size_t i = 0; i < v.size(); ++i) {
        PyObject *t = nullptr;
        if (v[i].defined()) t = THPVariable_Wrap(std::move(v[i]));
        else t = Py_NewRef(Py_None);
        if (!t) {
            Py_DECREF(l);
            return nullptr;
        }
        PyList_SET_ITEM(l, (Py_ssize_t)i, t);
    }
    return l;
}

// (first, list) with references stolen
PyObject *pair_of(PyObject *a, PyObject *b)
{
    PyObject *t = a && b ? PyTuple_New(2) : nullptr;
    if (!t) {
        Py_XDECREF(a);
        Py_XDECREF(b);
        return nullptr;
    }
    PyTuple_SET_ITEM(t, 0, a);
    PyTuple_SET_ITEM(t, 1, b);
    return t;
}

// run(x, residuals) -> (out, [index outputs]) or None
PyObject *plan_run(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 2) Py_RETURN_NONE;
    const std::shared_ptr<Plan> p = *reinterpret_cast<PlanObject *>(self)->plan;
    const at::Tensor *x;
    std::vector<at::Tensor> res, idx;
    if (!operands(*p, args[0], args[1], x, res)) Py_RETURN_NONE;
    const at::Tensor xs = *x;
    at::Tensor out;
    try {
        pybind11::gil_scoped_release no_gil;
        run_forward(*p, xs, res, out, idx);
    } catch (const CallFailed &e) {
        return failed(e);
    }
    return pair_of(THPVariable_Wrap(std::move(out)), wrap_list(idx));
    END_HANDLE_TH_ERRORS
}

// infer(x, residuals) -> out or None: as run, for plans without index outputs
PyObject *plan_infer(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 2) Py_RETURN_NONE;
    const std::shared_ptr<Plan> p = *reinterpret_cast<PlanObject *>(self)->plan;
    const at::Tensor *x;
    std::vector<at::Tensor> res, idx;
    if (!p->idx.empty() || !operands(*p, args[0], args[1], x, res)) Py_RETURN_NONE;
    const at::Tensor xs = *x;
    at::Tensor out;
    try {
        pybind11::gil_scoped_release no_gil;
        run_forward(*p, xs, res, out, idx);
    } catch (const CallFailed &e) {
        return failed(e);
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// backward(x, residuals, grad_out, indices or None) -> (grad_x, [residual gradients]) or None
PyObject *plan_backward(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 4) Py_RETURN_NONE;
    const std::shared_ptr<Plan> p = *reinterpret_cast<PlanObject *>(self)->plan;
    const at::Tensor *x;
    std::vector<at::Tensor> res, idx, gres;
    if (!p->bwd_planned || !operands(*p, args[0], args[1], x, res)) Py_RETURN_NONE;
    const at::Tensor *dy = tensor_of(args[2]);
    const at::Device dev = x->device();
    if (!dy || !plain(*p, *dy, p->out, p->dtype, &dev)) Py_RETURN_NONE;
    if (args[3] != Py_None) {
        if (!PyTuple_Check(args[3]) && !PyList_Check(args[3])) Py_RETURN_NONE;
        const Py_ssize_t m = PySequence_Fast_GET_SIZE(args[3]);
        if ((size_t)m != p->idx.size()) Py_RETURN_NONE;
        for (Py_ssize_t i = 0; i < m; ++i) {
            const at::Tensor *t = tensor_of(PySequence_Fast_GET_ITEM(args[3], i));
            if (!t || !plain(*p, *t, p->idx[i], at::kInt, &dev)) Py_RETURN_NONE;
            idx.push_back(*t);
        }
    }
    const at::Tensor xs = *x, dys = *dy;
    at::Tensor gx;
    try {
        pybind11::gil_scoped_release no_gil;
        run_backward(*p, xs, res, dys, 0, idx, std::vector<bool>(1 + res.size(), true), gx, gres);
    } catch (const CallFailed &e) {
        return failed(e);
    }
    return pair_of(THPVariable_Wrap(std::move(gx)), wrap_list(gres));
    END_HANDLE_TH_ERRORS
}

// record(x, residuals) -> out with its node in the autograd graph, or None
PyObject *plan_record(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 2) Py_RETURN_NONE;
    const std::shared_ptr<Plan> p = *reinterpret_cast<PlanObject *>(self)->plan;
    const at::Tensor *x;
    std::vector<at::Tensor> res;
    if (!p->bwd_planned || !operands(*p, args[0], args[1], x, res)) Py_RETURN_NONE;
    // forward-mode and functorch levels see the Python function's own answers
    if (x->_fw_grad(0).defined()) Py_RETURN_NONE;
    for (const at::Tensor &r : res)
        if (r._fw_grad(0).defined()) Py_RETURN_NONE;
    if (at::functorch::functorchTLSAccessor()) Py_RETURN_NONE;
    const at::Tensor xs = *x;
    try {
        return THPVariable_Wrap(StackNode::apply(p, xs, at::TensorList(res)));
    } catch (const CallFailed &e) {
        return failed(e);
    }
    END_HANDLE_TH_ERRORS
}

// set_backward(workspace bytes, reads picks): the backward pass is planned
PyObject *plan_set_backward(PyObject *self, PyObject *args)
{
    unsigned long long n;
    int reads;
    if (!PyArg_ParseTuple(args, "Kp", &n, &reads)) return nullptr;
    Plan &p = plan_of(self);
    {
        Plan::Buffers old;
        std::lock_guard<std::mutex> lock(p.mutex);
        p.bwd_ws_bytes = n;
        p.bwd_planned = true;
        p.bwd_reads_picks = reads != 0;
        old.swap(p.ws[1]);
    }
    Py_RETURN_NONE;
}

// workspace(backward?, device, raw stream) -> the buffer that calls on this stream hand intermediate tensors through, or None
PyObject *plan_workspace(PyObject *self, PyObject *args)
{
    HANDLE_TH_ERRORS
    int bwd;
    PyObject *dev;
    unsigned long long stream;
    if (!PyArg_ParseTuple(args, "pO!K", &bwd, &THPDeviceType, &dev, &stream)) return nullptr;
    const at::Tensor t = plan_of(self).workspace(bwd != 0, reinterpret_cast<THPDevice *>(dev)->device, reinterpret_cast<void *>(stream));
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
    END_HANDLE_TH_ERRORS
}

// release() -> handle: nothing runs through this object any more, and the caller destroys the handle (0: released before)
PyObject *plan_release(PyObject *self, PyObject *) { return PyLong_FromVoidPtr(plan_of(self).release()); }

PyObject *set_error(PyObject *, PyObject *cls)
{
    Py_XDECREF(g_error);
    g_error = Py_NewRef(cls);
    Py_RETURN_NONE;
}

// ---------------------------------------------------------------------------------------------------- operators without a plan
// Group normalisation and log probabilities (functional.py): the same bargain, every function returns None for what is not the plain case.  The
// tensors' device is the current one while a call runs: a default stream's handle names no device.
struct Operators {
    decltype(&bs_group_norm_workspace_bytes) norm_bytes;
    decltype(&bs_group_norm) norm;
    decltype(&bs_group_norm_backward) norm_backward;
    decltype(&bs_log_probs_workspace_bytes) head_bytes;
    decltype(&bs_log_probs) head;
    decltype(&bs_log_probs_backward) head_backward;
};
Operators g_operators{};

// set_operators((addresses of the six functions, in this order))
PyObject *set_operators(PyObject *, PyObject *args)
{
    unsigned long long a[6];
    if (!PyArg_ParseTuple(args, "(KKKKKK)", a, a + 1, a + 2, a + 3, a + 4, a + 5)) return nullptr;
    g_operators = {reinterpret_cast<decltype(Operators::norm_bytes)>(a[0]), reinterpret_cast<decltype(Operators::norm)>(a[1]),
                   reinterpret_cast<decltype(Operators::norm_backward)>(a[2]), reinterpret_cast<decltype(Operators::head_bytes)>(a[3]),
                   reinterpret_cast<decltype(Operators::head)>(a[4]), reinterpret_cast<decltype(Operators::head_backward)>(a[5])};
    Py_RETURN_NONE;
}

int32_t dtype_code(at::ScalarType t) { return t == at::kFloat ? BS_F32 : t == at::kBFloat16 ? BS_BF16 : t == at::kHalf ? BS_F16 : -1; }

// Whoever records, overrides or derives operations on tensors has to see the Python code's answer: torch.jit.trace, modes, forward-mode derivatives.
bool dual(const at::Tensor &t) { return t._fw_grad(0).defined(); }
bool recorders_active() { return modes_active() || at::impl::torch_function_mode_enabled() || torch::jit::tracer::isTracing(); }

// A tensor argument that may be None; false: neither (no error set), or one with a forward-mode derivative.
bool optional_tensor(PyObject *o, at::Tensor &t)
{
    if (o == Py_None) return true;
    const at::Tensor *p = tensor_of(o);
    if (!p) return false;
    t = *p;
    return t.defined() && !dual(t);
}
bool on_gpu(const at::Tensor &t, const at::Device &dev) { return t.is_cuda() && t.has_storage() && t.device() == dev; }

// Elements from a pixel to the next of a channels-last tensor or a channel slice of one; 0: it is neither.
int64_t pixel_stride(const at::Tensor &t)
{
    const int64_t n = t.size(0), c = t.size(1), h = t.size(2), w = t.size(3);
    const int64_t sn = t.stride(0), sc = t.stride(1), sh = t.stride(2), sw = t.stride(3);
    const int64_t step = w > 1 ? sw : h > 1 ? sh : n > 1 ? sn : c;
    return step >= c && (c == 1 || sc == 1) && (w == 1 || sw == step) && (h == 1 || sh == w * step) && (n == 1 || sn == h * w * step) ? step : 0;
}

bool read_int(PyObject *o, int64_t &v)
{
    v = PyLong_Check(o) ? PyLong_AsLongLong(o) : 0;
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return PyLong_Check(o);
}
bool read_float(PyObject *o, double &v)
{
    v = PyFloat_Check(o) ? PyFloat_AS_DOUBLE(o) : 0;
    return PyFloat_Check(o);
}

// The memory that the parts of an image hand their sums through: kept for every stream of torch's own (a device's default stream and its pools,
// which live as long as the process), zero-filled once.  (Never destroyed: the process may end after the device has gone.)
void *exchange_of(const at::Device &dev, const c10::hip::HIPStream &stream, const at::TensorOptions &like)
{
    // a recorded graph may run on any stream, next to later calls on this one: it gets none, and clears its workspace by a launch
    if (c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None) return nullptr;
    // so does a stream that torch did not make, whose id is its handle: a handle can stand for several streams (a thread's own default stream) or
    // come back for another one while the work of the first still runs
    const c10::StreamId id = stream.id();
    if (id != 0 && reinterpret_cast<void *>(id) == static_cast<void *>(stream.stream())) return nullptr;
    static std::mutex mutex;
    static auto &kept = *new std::map<std::pair<int, c10::StreamId>, at::Tensor>();
    const std::pair<int, c10::StreamId> key{dev.index(), id};
    {
        std::lock_guard<std::mutex> lock(mutex);
        const auto it = kept.find(key);
        if (it != kept.end()) return it->second.data_ptr();
    }
    const at::Tensor t = at::zeros({(int64_t)BS_GROUP_NORM_EXCHANGE_BYTES}, like.dtype(at::kByte));  // (outside the lock, as every allocation)
    std::lock_guard<std::mutex> lock(mutex);
    return kept.emplace(key, t).first->second.data_ptr();
}

struct NormCall {
    bs_group_norm_desc d{};
    at::Tensor x, weight, bias, residual;
    at::TensorOptions like;

    // x, groups, weight, bias, residual, activation, eps; false: not the plain case
    bool read(PyObject *xo, PyObject *groups, PyObject *wo, PyObject *bo, PyObject *ro, PyObject *act, PyObject *eps)
    {
        const at::Tensor *xp = tensor_of(xo);
        if (!g_operators.norm || !xp || recorders_active() || !xp->defined() || dual(*xp) || !xp->is_cuda() || !xp->has_storage() || xp->dim() != 4) return false;
        x = *xp;
        int64_t g, a;
        if (!read_int(groups, g) || !read_int(act, a) || !read_float(eps, d.eps) || g < 1 || g > x.size(1)) return false;
        if (!optional_tensor(wo, weight) || !optional_tensor(bo, bias) || !optional_tensor(ro, residual)) return false;
        d.groups = (int32_t)g;
        d.activation = (int32_t)a;
        d.dtype = dtype_code(x.scalar_type());
        d.param_dtype = BS_F32;
        for (int i = 0; i < 4; ++i) d.shape[i] = x.size(i);
        if (d.dtype < 0 || x.size(0) < 1 || (d.x_stride = pixel_stride(x)) == 0) return false;
        like = x.options();
        at::ScalarType type = at::ScalarType::Undefined;
        for (const at::Tensor *p : {&weight, &bias}) {
            if (!p->defined()) continue;
            if (!on_gpu(*p, x.device()) || p->dim() != 1 || p->size(0) != x.size(1) || !p->is_contiguous()) return false;
            if (p->scalar_type() != at::kFloat && p->scalar_type() != x.scalar_type()) return false;
            if (type != at::ScalarType::Undefined && type != p->scalar_type()) return false;
            type = p->scalar_type();
            d.param_dtype = dtype_code(type);
        }
        return beside(residual, d.residual_stride);
    }
    // A tensor of x's shape, type and device that is read in place (or none).
    bool beside(const at::Tensor &t, int64_t &stride) const
    {
        return !t.defined() || (on_gpu(t, x.device()) && t.sizes() == x.sizes() && t.scalar_type() == x.scalar_type() && (stride = pixel_stride(t)) != 0);
    }
    at::Tensor empty() const { return at::empty(x.sizes(), like.memory_format(at::MemoryFormat::ChannelsLast)); }
    // Small images are one part and need none.
    void exchange(const c10::hip::HIPStream &stream)
    {
        if (d.shape[1] * d.shape[2] * d.shape[3] < 8192) return;
        d.exchange = exchange_of(x.device(), stream, like);
        d.exchange_bytes = d.exchange ? BS_GROUP_NORM_EXCHANGE_BYTES : 0;
    }
    static void *ptr(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
};

at::Tensor workspace_of(uint64_t n, const at::TensorOptions &like)
{
    return n ? at::empty({(int64_t)n}, like.dtype(at::kByte)) : at::Tensor();
}

PyObject *tuple_of(std::initializer_list<at::Tensor> tensors)
{
    PyObject *t = PyTuple_New((Py_ssize_t)tensors.size());
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor &v : tensors) {
        PyObject *o = v.defined() ? THPVariable_Wrap(v) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}

// group_norm(x, groups, weight, bias, residual, activation, eps, keep statistics?) -> y, (y, stats) or None
PyObject *group_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    NormCall c;
    if (n != 8 || !c.read(args[0], args[1], args[2], args[3], args[4], args[5], args[6])) Py_RETURN_NONE;
    const bool keep = args[7] == Py_True;
    at::Tensor y, stats;
    try {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(c.x.device());
        y = c.empty();
        if (keep) stats = at::empty({c.x.size(0), c.d.groups, 2}, c.like.dtype(at::kFloat));
        const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream(c.x.device().index());
        c.exchange(stream);
        const uint64_t bytes = g_operators.norm_bytes(&c.d, 0);
        const at::Tensor ws = workspace_of(bytes, c.like);
        const int rc = g_operators.norm(&c.d, c.x.data_ptr(), c.ptr(c.residual), c.ptr(c.weight), c.ptr(c.bias), y.data_ptr(), static_cast<float *>(c.ptr(stats)),
                                        c.ptr(ws), bytes, stream.stream());
        if (rc != 0) throw CallFailed(rc, "bs_group_norm");
    } catch (const CallFailed &e) {
        return failed(e);
    }
    return keep ? tuple_of({y, stats}) : THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

// group_norm_backward(x, stats, grad, groups, weight, bias, residual, activation, eps, wanted: bits 1 x, 2 weight, 4 bias, 8 residual)
// -> (grad_x, grad_weight, grad_bias, grad_residual) or None
PyObject *group_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    NormCall c;
    if (n != 10 || !c.read(args[0], args[3], args[4], args[5], args[6], args[7], args[8])) Py_RETURN_NONE;
    const at::Tensor *stats = tensor_of(args[1]), *grad = tensor_of(args[2]);
    int64_t wanted;
    if (!stats || !grad || !stats->defined() || !grad->defined() || dual(*stats) || dual(*grad) || !read_int(args[9], wanted) || !c.beside(*grad, c.d.grad_y_stride)) Py_RETURN_NONE;
    if (!on_gpu(*stats, c.x.device()) || stats->scalar_type() != at::kFloat || !stats->is_contiguous() || stats->dim() != 3 || stats->size(0) != c.x.size(0) ||
        stats->size(1) != c.d.groups || stats->size(2) != 2)
        Py_RETURN_NONE;
    const at::Tensor st = *stats, dy = *grad;
    at::Tensor gx, gw, gb, gr;
    try {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(c.x.device());
        if (wanted & 1) gx = c.empty();
        if ((wanted & 2) && c.weight.defined()) gw = at::empty({c.x.size(1)}, c.weight.options());
        if ((wanted & 4) && c.bias.defined()) gb = at::empty({c.x.size(1)}, c.bias.options());
        if ((wanted & 8) && c.residual.defined()) gr = c.empty();
        const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream(c.x.device().index());
        c.exchange(stream);
        const uint64_t bytes = g_operators.norm_bytes(&c.d, 1);
        const at::Tensor ws = workspace_of(bytes, c.like);
        const int rc = g_operators.norm_backward(&c.d, c.x.data_ptr(), c.ptr(c.residual), c.ptr(c.weight), c.ptr(c.bias), static_cast<const float *>(st.data_ptr()),
                                                 dy.data_ptr(), c.ptr(gx), c.ptr(gr), c.ptr(gw), c.ptr(gb), c.ptr(ws), bytes, stream.stream());
        if (rc != 0) throw CallFailed(rc, "bs_group_norm_backward");
    } catch (const CallFailed &e) {
        return failed(e);
    }
    return tuple_of({gx, gw, gb, gr});
    END_HANDLE_TH_ERRORS
}

struct HeadCall {
    bs_log_probs_desc d{};
    at::Tensor logits, targets;

    // Elements from a row to the next where the classes of a row are contiguous; -1: they are not.
    static int64_t row_stride(const at::Tensor &t)
    {
        const int64_t rows = t.size(0), classes = t.size(1);
        if ((classes > 1 && t.stride(1) != 1) || (rows > 1 && t.stride(0) < classes)) return -1;
        return rows > 1 ? t.stride(0) : classes;
    }
    bool read(PyObject *lo, PyObject *to, PyObject *top, PyObject *ignore)
    {
        const at::Tensor *lp = tensor_of(lo);
        if (!g_operators.head || !lp || recorders_active() || !lp->defined() || dual(*lp) || !lp->is_cuda() || !lp->has_storage() || lp->dim() != 2) return false;
        logits = *lp;
        int64_t k;
        if (!optional_tensor(to, targets) || !read_int(top, k) || k < 0 || k > BS_MAX_TOP || !read_int(ignore, d.ignore_index)) return false;
        d.rows = logits.size(0);
        d.classes = logits.size(1);
        d.top = (int32_t)k;
        d.dtype = dtype_code(logits.scalar_type());
        d.target_bytes = d.lse_bytes = 8;
        if (d.dtype < 0 || d.rows < 1 || d.classes < 1 || (d.row_stride = row_stride(logits)) < 0) return false;
        if (targets.defined()) {
            if (!on_gpu(targets, logits.device()) || targets.dim() != 1 || targets.size(0) != d.rows || !targets.is_contiguous()) return false;
            if (targets.scalar_type() != at::kLong && targets.scalar_type() != at::kInt) return false;
            d.target_bytes = targets.scalar_type() == at::kInt ? 4 : 8;
        }
        return true;
    }
    bool per_row(const at::Tensor &t, at::ScalarType type = at::kFloat) const
    {
        return !t.defined() || (on_gpu(t, logits.device()) && t.scalar_type() == type && t.dim() == 1 && t.size(0) == d.rows && t.is_contiguous());
    }
};

// log_probs(logits, targets, top, ignore_index) -> (logp, entropy, top_logp, top_index, lse) or None
PyObject *log_probs(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    HeadCall c;
    if (n != 4 || !c.read(args[0], args[1], args[2], args[3])) Py_RETURN_NONE;
    at::Tensor logp, entropy, lse, top_logp, top_index;
    try {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(c.logits.device());
        const at::TensorOptions f32 = c.logits.options().dtype(at::kFloat);
        if (c.targets.defined()) logp = at::empty({c.d.rows}, f32);
        entropy = at::empty({c.d.rows}, f32);
        lse = at::empty({c.d.rows}, f32.dtype(at::kDouble));
        if (c.d.top) {
            top_logp = at::empty({c.d.rows, c.d.top}, f32);
            top_index = at::empty({c.d.rows, c.d.top}, f32.dtype(at::kInt));
        }
        const uint64_t bytes = g_operators.head_bytes(&c.d);
        const at::Tensor ws = workspace_of(bytes, f32);
        auto p = [](const at::Tensor &t) { return static_cast<float *>(NormCall::ptr(t)); };
        const int rc = g_operators.head(&c.d, c.logits.data_ptr(), NormCall::ptr(c.targets), p(logp), p(entropy), NormCall::ptr(lse), p(top_logp),
                                        static_cast<int32_t *>(NormCall::ptr(top_index)), NormCall::ptr(ws), bytes,
                                        c10::hip::getCurrentHIPStream(c.logits.device().index()).stream());
        if (rc != 0) throw CallFailed(rc, "bs_log_probs");
    } catch (const CallFailed &e) {
        return failed(e);
    }
    return tuple_of({logp, entropy, top_logp, top_index, lse});
    END_HANDLE_TH_ERRORS
}

// log_probs_backward(logits, targets, lse, entropy, grad_logp, grad_entropy, ignore_index) -> grad_logits or None
PyObject *log_probs_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    HeadCall c;
    at::Tensor lse, entropy, g, h, out;
    PyObject *const zero = PyLong_FromLong(0);
    const bool fits = n == 7 && c.read(args[0], args[1], zero, args[6]) && optional_tensor(args[2], lse) && optional_tensor(args[3], entropy) &&
                      optional_tensor(args[4], g) && optional_tensor(args[5], h);
    Py_XDECREF(zero);
    if (!fits || !lse.defined() || !c.per_row(lse, at::kDouble) || !c.per_row(entropy) || !c.per_row(g) || !c.per_row(h)) Py_RETURN_NONE;
    try {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(c.logits.device());
        out = at::empty({c.d.rows, c.d.classes}, c.logits.options());
        auto p = [](const at::Tensor &t) { return static_cast<const float *>(NormCall::ptr(t)); };
        const int rc = g_operators.head_backward(&c.d, c.logits.data_ptr(), NormCall::ptr(c.targets), NormCall::ptr(lse), p(entropy), p(g), p(h), out.data_ptr(),
                                                 c10::hip::getCurrentHIPStream(c.logits.device().index()).stream());
        if (rc != 0) throw CallFailed(rc, "bs_log_probs_backward");
    } catch (const CallFailed &e) {
        return failed(e);
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

template <typename F>
constexpr PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef plan_methods[] = {
    {"run", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(plan_run)), METH_FASTCALL, "(x, residuals) -> (out, indices) or None"},
    {"infer", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(plan_infer)), METH_FASTCALL, "(x, residuals) -> out or None"},
    {"backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(plan_backward)), METH_FASTCALL,
     "(x, residuals, grad_out, indices or None) -> (grad_x, residual gradients) or None"},
    {"record", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(plan_record)), METH_FASTCALL, "(x, residuals) -> out in the autograd graph, or None"},
    {"set_backward", plan_set_backward, METH_VARARGS, "(workspace bytes, reads picks)"},
    {"workspace", plan_workspace, METH_VARARGS, "(backward, device, raw stream) -> buffer or None"},
    {"release", plan_release, METH_NOARGS, "-> handle"},
    {nullptr, nullptr, 0, nullptr}};

PyType_Slot plan_slots[] = {{Py_tp_new, reinterpret_cast<void *>(plan_new)},
                            {Py_tp_dealloc, reinterpret_cast<void *>(plan_dealloc)},
                            {Py_tp_methods, plan_methods},
                            {0, nullptr}};
PyType_Spec plan_spec = {"_bs_torch.Plan", sizeof(PlanObject), 0, Py_TPFLAGS_DEFAULT, plan_slots};

PyMethodDef module_methods[] = {{"set_error", set_error, METH_O, "(class): raised as class(status, where)"},
                                {"set_operators", set_operators, METH_VARARGS, "((addresses,)): the library's functions without a plan"},
                                {"group_norm", fast(group_norm), METH_FASTCALL, "(x, groups, weight, bias, residual, activation, eps, keep) -> y, (y, stats) or None"},
                                {"group_norm_backward", fast(group_norm_backward), METH_FASTCALL,
                                 "(x, stats, grad, groups, weight, bias, residual, activation, eps, wanted) -> gradients or None"},
                                {"log_probs", fast(log_probs), METH_FASTCALL, "(logits, targets, top, ignore_index) -> results or None"},
                                {"log_probs_backward", fast(log_probs_backward), METH_FASTCALL,
                                 "(logits, targets, lse, entropy, grad_logp, grad_entropy, ignore_index) -> gradient or None"},
                                {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_bs_torch", nullptr, -1, module_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: what the file was compiled for; read from the file before it is loaded
extern "C" __attribute__((visibility("default"))) PyObject *PyInit__bs_torch(void)
{
    PyObject *m = PyModule_Create(&module_def);
    if (!m) return nullptr;
    PyObject *t = PyType_FromSpec(&plan_spec);
    if (!t || PyModule_AddStringConstant(m, "built_for", BS_TORCH_TAG) != 0 || PyModule_AddObject(m, "Plan", t) != 0) {
        Py_XDECREF(t);
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
