// The plain calls of the Python binding in native code: checks, allocation of the outputs and of the workspace, launch.
//
// One image through a small layer, or a network of small blocks, is bound by the host.  us per call on the host, through ctypes -> here:
// scc_forward 7.7 -> 4.5 (its launch: 3.6), scc_backward 10.5 -> 5.9, scc_dw_backward 21 -> 11; a training step of the 13-block stack at
// batch 128 925 -> 709 (then bound by its kernels), its forward at batch 16 145 -> 114, one 8x8 image forward and backward 18.6 -> 11.6.
// Each function here serves the call that a program makes all day (dense,
// contiguous tensors of the right shapes on the current device, no `out`, no workspace, no modes) and returns None for
// everything else, errors included: scc.py then goes its general way, which raises what there is to raise (orthogonal_step, which moves
// its arguments, answers a failed call's status instead).  Nothing is kept from one call to the next.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <ATen/ops/zeros_like.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>

#include "scc.h"

namespace {

// A dense contiguous tensor on the current device in one of the library's types (and, for the second overload, those of x).
bool plain(const at::Tensor& t)
{
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && t.is_contiguous() &&
           (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16) &&
           t.get_device() == c10::hip::current_device();
}

bool plain(const at::Tensor& t, const at::Tensor& x) { return plain(t) && t.scalar_type() == x.scalar_type(); }

bool fits(const at::Tensor& t)
{
    for (const int64_t s : t.sizes())
        if (s < 1 || s > INT_MAX) return false;
    return true;
}

// Arguments of a call: `tensors` tensors that are no subclass (Parameter aside), cg, co and, with `strided`, the stage's stride.
struct Args {
    const at::Tensor* t[4];
    int cg, stride;
    double co;
};

bool integer(PyObject* o, int* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long l = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || l < 1 || l > INT_MAX) return false;
    *v = (int)l;
    return true;
}

bool parse(PyObject* const* a, Py_ssize_t n, int tensors, bool strided, Args* out)
{
    if (n != tensors + 2 + (strided ? 1 : 0)) return false;
    if (c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::PythonTorchFunctionTLS::stack_len() > 0) return false;
    for (int i = 0; i < tensors; ++i) {
        if (!THPVariable_CheckExact(a[i])) return false;
        out->t[i] = &THPVariable_Unpack(a[i]);
    }
    out->stride = 1;
    if (!integer(a[tensors], &out->cg) || (strided && !integer(a[tensors + 2], &out->stride))) return false;
    if (!PyFloat_CheckExact(a[tensors + 1])) return false;
    out->co = PyFloat_AS_DOUBLE(a[tensors + 1]);
    return true;
}

// x [N,Cin,H,W] and w [Cout,Cin/cg] as a layer; the map behind a depthwise stage of the given stride is Ho x Wo.
struct Layer {
    int N, Cin, Cout, H, W, Ho, Wo;
    scc_dtype dtype;
};

bool layer(const Args& a, const at::Tensor& x, const at::Tensor& w, Layer* l)
{
    if (!plain(x) || !plain(w, x) || x.dim() != 4 || w.dim() != 2 || !fits(x) || !fits(w)) return false;
    l->N = (int)x.size(0);
    l->Cin = (int)x.size(1);
    l->Cout = (int)w.size(0);
    l->H = (int)x.size(2);
    l->W = (int)x.size(3);
    l->Ho = (l->H - 1) / a.stride + 1;
    l->Wo = (l->W - 1) / a.stride + 1;
    l->dtype = x.scalar_type() == at::kFloat ? SCC_F32 : SCC_BF16;
    return l->Cin % a.cg == 0 && w.size(1) == l->Cin / a.cg;
}

bool taps(const at::Tensor& k, const at::Tensor& x, const Layer& l)
{
    return plain(k, x) && k.dim() == 3 && k.size(0) == l.Cin && k.size(1) == 3 && k.size(2) == 3;
}

bool outputs(const at::Tensor& g, const at::Tensor& x, const Layer& l)
{
    return plain(g, x) && g.dim() == 4 && g.size(0) == l.N && g.size(1) == l.Cout && g.size(2) == l.Ho && g.size(3) == l.Wo;
}

at::Tensor scratch(size_t need, const at::Tensor& x)
{
    return need ? at::empty({(int64_t)need}, x.options().dtype(at::kByte)) : at::Tensor();
}

void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// f(stream) without the interpreter's lock, as a call through ctypes runs
struct Unlocked {
    PyThreadState* save = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(save); }
};

void* stream_of(const at::Tensor& x) { return (void*)c10::hip::getCurrentHIPStream(x.get_device()).stream(); }

template <typename F>
int launch(const at::Tensor& x, F&& f)
{
    void* stream = stream_of(x);
    Unlocked unlocked;
    return f(stream);
}

PyObject* tuple_of(std::initializer_list<at::Tensor> ts)
{
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    if (r)
        for (const at::Tensor& t : ts) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
    return r;
}

PyObject* forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    if (!parse(args, n, 2, false, &a) || !layer(a, *a.t[0], *a.t[1], &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &w = *a.t[1];
    at::Tensor y = at::empty({l.N, l.Cout, l.H, l.W}, x.options());
    const size_t need = scc_forward_workspace_bytes(l.N, l.Cin, l.Cout, l.H, l.W, a.cg, a.co, l.dtype);
    const at::Tensor ws = scratch(need, x);
    const int rc = launch(x, [&](void* st) {
        return scc_forward_ws(x.data_ptr(), w.data_ptr(), y.data_ptr(), l.N, l.Cin, l.Cout, l.H, l.W, a.cg, a.co, l.dtype,
                              address(ws), need, st);
    });
    if (rc != SCC_OK) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

PyObject* backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    if (!parse(args, n, 3, false, &a) || !layer(a, *a.t[0], *a.t[2], &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &dy = *a.t[1], &w = *a.t[2];
    if (!outputs(dy, x, l)) Py_RETURN_NONE;
    at::Tensor dx = at::empty_like(x), dw = at::empty(w.sizes(), x.options().dtype(at::kFloat));
    const size_t need = scc_backward_workspace_bytes(l.N, l.Cin, l.Cout, l.H, l.W, a.cg, a.co, l.dtype);
    const at::Tensor ws = scratch(need, x);
    const int rc = launch(x, [&](void* st) {
        return scc_backward(x.data_ptr(), dy.data_ptr(), w.data_ptr(), dx.data_ptr(), dw.data_ptr(), l.N, l.Cin, l.Cout, l.H, l.W,
                            a.cg, a.co, l.dtype, address(ws), need, st);
    });
    if (rc != SCC_OK) Py_RETURN_NONE;
    return tuple_of({dx, dw});
    END_HANDLE_TH_ERRORS
}

// y of a block; undefined where the call failed
template <typename F>
at::Tensor block_forward(const at::Tensor& x, const at::Tensor& k, const at::Tensor& w, const Args& a, const Layer& l, F&& run)
{
    at::Tensor y = at::empty({l.N, l.Cout, l.Ho, l.Wo}, x.options());
    const size_t need = scc_dw_forward_workspace_bytes(l.N, l.Cin, l.Cout, l.H, l.W, a.stride, a.cg, a.co, l.dtype);
    const at::Tensor ws = scratch(need, x);
    const int rc = run([&](void* st) {
        return scc_dw_forward_scratch(x.data_ptr(), k.data_ptr(), w.data_ptr(), y.data_ptr(), l.N, l.Cin, l.Cout, l.H, l.W,
                                      a.stride, a.cg, a.co, l.dtype, address(ws), need, st);
    });
    return rc == SCC_OK ? y : at::Tensor();
}

// dx, dkdw, dw of a block; none where the call failed
template <typename F>
std::vector<at::Tensor> block_backward(const at::Tensor& x, const at::Tensor& k, const at::Tensor& w, const at::Tensor& dy,
                                       const Args& a, const Layer& l, scc_dtype grad, F&& run)
{
    const at::TensorOptions of = x.options().dtype(grad == SCC_F32 ? at::kFloat : at::kBFloat16);
    at::Tensor dx = at::empty_like(x), dk = at::empty(k.sizes(), of), dw = at::empty(w.sizes(), of);
    const size_t need = scc_dw_backward_as_workspace_bytes(l.N, l.Cin, l.Cout, l.H, l.W, a.stride, a.cg, a.co, l.dtype, grad);
    const at::Tensor ws = scratch(need, x);
    const int rc = run([&](void* st) {
        return scc_dw_backward_as(x.data_ptr(), k.data_ptr(), w.data_ptr(), dy.data_ptr(), dx.data_ptr(), dk.data_ptr(),
                                  dw.data_ptr(), l.N, l.Cin, l.Cout, l.H, l.W, a.stride, a.cg, a.co, l.dtype, grad, address(ws), need,
                                  st);
    });
    if (rc != SCC_OK) return {};
    return {dx, dk, dw};
}

PyObject* dw_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    if (!parse(args, n, 3, true, &a) || !layer(a, *a.t[0], *a.t[2], &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &k = *a.t[1], &w = *a.t[2];
    if (!taps(k, x, l)) Py_RETURN_NONE;
    at::Tensor y = block_forward(x, k, w, a, l, [&](auto&& f) { return launch(x, f); });
    if (!y.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

PyObject* dw_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    if (n != 8 || !PyBool_Check(args[7]) || !parse(args, 7, 4, true, &a) || !layer(a, *a.t[0], *a.t[2], &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &k = *a.t[1], &w = *a.t[2], &dy = *a.t[3];
    if (!taps(k, x, l) || !outputs(dy, x, l)) Py_RETURN_NONE;
    const std::vector<at::Tensor> g = block_backward(x, k, w, dy, a, l, args[7] == Py_True ? l.dtype : SCC_F32,
                                                     [&](auto&& f) { return launch(x, f); });
    if (g.empty()) Py_RETURN_NONE;
    return tuple_of({g[0], g[1], g[2]});
    END_HANDLE_TH_ERRORS
}

// nn._FirstOrder: gradients under create_graph, which only differentiating them makes an error of
struct FirstOrder : torch::autograd::Function<FirstOrder> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext*, const at::Tensor& dx, const at::Tensor& dk,
                                                  const at::Tensor& dw, const at::Tensor&, const at::Tensor&, const at::Tensor&,
                                                  const at::Tensor&)
    {
        return {dx.detach(), dk.detach(), dw.detach()};
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext*, torch::autograd::variable_list)
    {
        TORCH_CHECK(false, "this operator has no second derivative");
    }
};

// A block under autograd: nn.DWSCCFunction for the training step of a plain call, all of whose tensors want gradients.  Through the Python function
// a block costs 40 us of host time more, forward and backward, than its launches take (128 x 128 -> 256 on 32x32, stride 2, bf16, one
// step: 95 us of which the kernels are 62).
struct Block : torch::autograd::Function<Block> {
    struct Refused {};

    // from a call of the interpreter, whose lock is held
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& k, const at::Tensor& w,
                              int64_t cg, double co, int64_t stride)
    {
        const Args a = {{&x, &k, &w, nullptr}, (int)cg, (int)stride, co};
        Layer l;
        at::Tensor y;
        if (layer(a, x, w, &l)) y = block_forward(x, k, w, a, l, [&](auto&& f) { return launch(x, f); });
        if (!y.defined()) throw Refused();
        ctx->save_for_backward({x, k, w});
        ctx->saved_data["cg"] = cg;
        ctx->saved_data["co"] = co;
        ctx->saved_data["stride"] = stride;
        return y;
    }

    // The engine's thread: the interpreter's lock is not held.
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const torch::autograd::variable_list saved = ctx->get_saved_variables();
        const at::Tensor &x = saved[0], &k = saved[1], &w = saved[2];
        const at::Tensor dy = grads[0].contiguous();
        Args a = {{&x, &k, &w, &dy}, (int)ctx->saved_data["cg"].toInt(), (int)ctx->saved_data["stride"].toInt(),
                  ctx->saved_data["co"].toDouble()};
        Layer l;
        std::vector<at::Tensor> g;
        if (layer(a, x, w, &l) && taps(k, x, l) && outputs(dy, x, l))
            g = block_backward(x, k, w, dy, a, l, l.dtype, [&](auto&& f) { return f(stream_of(x)); });
        if (g.empty()) g = general(a);
        if (at::GradMode::is_enabled()) g = FirstOrder::apply(g[0], g[1], g[2], x, k, w, dy);
        return {g[0], g[1], g[2], at::Tensor(), at::Tensor(), at::Tensor()};
    }

    // what is not plain any more (tensors that saved-tensor hooks brought back, say), and errors: scc._dw_backward
    static std::vector<at::Tensor> general(const Args& a)
    {
        struct Locked {
            PyGILState_STATE s = PyGILState_Ensure();
            ~Locked() { PyGILState_Release(s); }
        } locked;
        std::vector<at::Tensor> g;
        PyObject* m = PyImport_ImportModule("paper_2101_00745_amd.scc");
        PyObject* t[4] = {};
        for (int i = 0; i < 4; ++i) t[i] = THPVariable_Wrap(*a.t[i]);
        PyObject* r = m ? PyObject_CallMethod(m, "_dw_backward", "OOOOidiO", t[0], t[1], t[2], t[3], a.cg, a.co, a.stride, Py_True) : nullptr;
        for (int i = 0; r && i < 3; ++i) g.push_back(THPVariable_Unpack(PyTuple_GetItem(r, i)));
        for (int i = 0; i < 4; ++i) Py_XDECREF(t[i]);
        Py_XDECREF(r);
        Py_XDECREF(m);
        if (!r) {
            python_error e;
            e.persist();
            throw e;
        }
        return g;
    }
};

PyObject* dw_block(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    if (!at::GradMode::is_enabled() || !parse(args, n, 3, true, &a) || !layer(a, *a.t[0], *a.t[2], &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &k = *a.t[1], &w = *a.t[2];
    if (!taps(k, x, l)) Py_RETURN_NONE;
    for (int i = 0; i < 3; ++i)
        if (!a.t[i]->requires_grad() || a.t[i]->is_inference() || a.t[i]->_fw_grad(0).defined()) Py_RETURN_NONE;
    try {
        return THPVariable_Wrap(Block::apply(x, k, w, (int64_t)a.cg, a.co, (int64_t)a.stride));
    } catch (const Block::Refused&) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}

// x [N,Cin,H,W], w [2,Cout,Cin/cg], cg, co and the activation's code of a gated layer's call, dy behind w where there is one
bool gated(PyObject* const* args, int tensors, Args* a, int* act, Layer* l)
{
    if (!PyLong_CheckExact(args[tensors + 2]) || !parse(args, tensors + 2, tensors, false, a)) return false;
    *act = (int)PyLong_AsLong(args[tensors + 2]);
    const at::Tensor &x = *a->t[0], &w = *a->t[1];
    return w.dim() == 3 && w.size(0) == 2 && w.is_contiguous() && layer(*a, x, w.select(0, 0), l);
}

template <typename F>
at::Tensor gated_forward_of(const at::Tensor& x, const at::Tensor& w, const Args& a, int act, const Layer& l, F&& run)
{
    at::Tensor y = at::empty({l.N, l.Cout, l.H, l.W}, x.options());
    const size_t need = scc_gated_forward_workspace_bytes(l.N, l.Cin, l.Cout, l.H, l.W, a.cg, a.co, l.dtype);
    const at::Tensor ws = scratch(need, x);
    const int rc = run([&](void* st) {
        return scc_gated_forward(x.data_ptr(), w.data_ptr(), y.data_ptr(), l.N, l.Cin, l.Cout, l.H, l.W, a.cg, a.co,
                                 (scc_activation)act, l.dtype, address(ws), need, st);
    });
    return rc == SCC_OK ? y : at::Tensor();
}

// dx, dw; none where the call failed
template <typename F>
std::vector<at::Tensor> gated_backward_of(const at::Tensor& x, const at::Tensor& w, const at::Tensor& dy, const Args& a, int act,
                                          const Layer& l, scc_dtype grad, F&& run)
{
    at::Tensor dx = at::empty_like(x);
    at::Tensor dw = at::empty(w.sizes(), x.options().dtype(grad == SCC_F32 ? at::kFloat : at::kBFloat16));
    const size_t need = scc_gated_backward_workspace_bytes(l.N, l.Cin, l.Cout, l.H, l.W, a.cg, a.co, l.dtype, grad);
    const at::Tensor ws = scratch(need, x);
    const int rc = run([&](void* st) {
        return scc_gated_backward(x.data_ptr(), w.data_ptr(), dy.data_ptr(), dx.data_ptr(), dw.data_ptr(), l.N, l.Cin, l.Cout, l.H,
                                  l.W, a.cg, a.co, (scc_activation)act, l.dtype, grad, address(ws), need, st);
    });
    if (rc != SCC_OK) return {};
    return {dx, dw};
}

PyObject* gated_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    int act;
    if (n != 5 || !gated(args, 2, &a, &act, &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &w = *a.t[1];
    at::Tensor y = gated_forward_of(x, w, a, act, l, [&](auto&& f) { return launch(x, f); });
    if (!y.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

PyObject* gated_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    int act;
    if (n != 7 || !PyBool_Check(args[6]) || !gated(args, 3, &a, &act, &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &w = *a.t[1], &dy = *a.t[2];
    if (!outputs(dy, x, l)) Py_RETURN_NONE;
    const std::vector<at::Tensor> g = gated_backward_of(x, w, dy, a, act, l, args[6] == Py_True ? l.dtype : SCC_F32,
                                                        [&](auto&& f) { return launch(x, f); });
    if (g.empty()) Py_RETURN_NONE;
    return tuple_of({g[0], g[1]});
    END_HANDLE_TH_ERRORS
}

struct FirstOrderPair : torch::autograd::Function<FirstOrderPair> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext*, const at::Tensor& dx, const at::Tensor& dw,
                                                  const at::Tensor&, const at::Tensor&, const at::Tensor&)
    {
        return {dx.detach(), dw.detach()};
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext*, torch::autograd::variable_list)
    {
        TORCH_CHECK(false, "this operator has no second derivative");
    }
};

// nn.GatedSCCFunction for a plain call whose two tensors want gradients, as Block is nn.DWSCCFunction
struct Gated : torch::autograd::Function<Gated> {
    struct Refused {};

    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w, int64_t cg, double co,
                              int64_t act)
    {
        const Args a = {{&x, &w, nullptr, nullptr}, (int)cg, 1, co};
        Layer l;
        at::Tensor y;
        if (layer(a, x, w.select(0, 0), &l)) y = gated_forward_of(x, w, a, (int)act, l, [&](auto&& f) { return launch(x, f); });
        if (!y.defined()) throw Refused();
        ctx->save_for_backward({x, w});
        ctx->saved_data["cg"] = cg;
        ctx->saved_data["co"] = co;
        ctx->saved_data["act"] = act;
        return y;
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const torch::autograd::variable_list saved = ctx->get_saved_variables();
        const at::Tensor &x = saved[0], &w = saved[1];
        const at::Tensor dy = grads[0].contiguous();
        const Args a = {{&x, &w, &dy, nullptr}, (int)ctx->saved_data["cg"].toInt(), 1, ctx->saved_data["co"].toDouble()};
        const int act = (int)ctx->saved_data["act"].toInt();
        Layer l;
        std::vector<at::Tensor> g;
        if (w.dim() == 3 && w.is_contiguous() && layer(a, x, w.select(0, 0), &l) && outputs(dy, x, l))
            g = gated_backward_of(x, w, dy, a, act, l, l.dtype, [&](auto&& f) { return f(stream_of(x)); });
        if (g.empty()) g = general(a, act);
        if (at::GradMode::is_enabled()) g = FirstOrderPair::apply(g[0], g[1], x, w, dy);
        return {g[0], g[1], at::Tensor(), at::Tensor(), at::Tensor()};
    }

    static std::vector<at::Tensor> general(const Args& a, int act)
    {
        struct Locked {
            PyGILState_STATE s = PyGILState_Ensure();
            ~Locked() { PyGILState_Release(s); }
        } locked;
        std::vector<at::Tensor> g;
        PyObject* m = PyImport_ImportModule("paper_2101_00745_amd.scc");
        PyObject* t[3] = {};
        for (int i = 0; i < 3; ++i) t[i] = THPVariable_Wrap(*a.t[i]);
        PyObject* r = m ? PyObject_CallMethod(m, "_gated_backward", "OOOidiO", t[0], t[1], t[2], a.cg, a.co, act, Py_True) : nullptr;
        for (int i = 0; r && i < 2; ++i) g.push_back(THPVariable_Unpack(PyTuple_GetItem(r, i)));
        for (int i = 0; i < 3; ++i) Py_XDECREF(t[i]);
        Py_XDECREF(r);
        Py_XDECREF(m);
        if (!r) {
            python_error e;
            e.persist();
            throw e;
        }
        return g;
    }
};

PyObject* gated_block(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a;
    Layer l;
    int act;
    if (n != 5 || !at::GradMode::is_enabled() || !gated(args, 2, &a, &act, &l)) Py_RETURN_NONE;
    const at::Tensor &x = *a.t[0], &w = *a.t[1];
    for (int i = 0; i < 2; ++i)
        if (!a.t[i]->requires_grad() || a.t[i]->is_inference() || a.t[i]->_fw_grad(0).defined()) Py_RETURN_NONE;
    try {
        return THPVariable_Wrap(Gated::apply(x, w, (int64_t)a.cg, a.co, (int64_t)act));
    } catch (const Gated::Refused&) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}

// A list of plain matrices of one type.
bool matrices(PyObject* o, Py_ssize_t count, at::ScalarType type, std::vector<const at::Tensor*>* out)
{
    if (!PyList_CheckExact(o) || PyList_GET_SIZE(o) != count) return false;
    for (Py_ssize_t i = 0; i < count; ++i) {
        PyObject* e = PyList_GET_ITEM(o, i);
        if (!THPVariable_CheckExact(e)) return false;
        const at::Tensor& t = THPVariable_Unpack(e);
        if (!plain(t) || t.dim() != 2 || t.scalar_type() != type || !fits(t)) return false;
        out->push_back(&t);
    }
    return true;
}

// A list's addresses and sizes, as the library takes them
struct List {
    std::vector<void*> address;
    std::vector<int> rows, cols;
    size_t need;
    at::Tensor ws;
};

bool begin_list(PyObject* first, std::vector<const at::Tensor*>* ts, List* l)
{
    if (c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::PythonTorchFunctionTLS::stack_len() > 0) return false;
    if (!PyList_CheckExact(first) || PyList_GET_SIZE(first) < 1 || PyList_GET_SIZE(first) > INT_MAX) return false;
    PyObject* e = PyList_GET_ITEM(first, 0);
    if (!THPVariable_CheckExact(e)) return false;
    if (!matrices(first, PyList_GET_SIZE(first), THPVariable_Unpack(e).scalar_type(), ts)) return false;
    for (const at::Tensor* t : *ts) {
        l->address.push_back(t->data_ptr());
        l->rows.push_back((int)t->size(0));
        l->cols.push_back((int)t->size(1));
    }
    l->need = scc_orthogonal_workspace_bytes((int)ts->size(), l->rows.data(), l->cols.data());
    if (l->need) l->ws = scratch(l->need, *(*ts)[0]);
    return l->need != 0;
}

bool numbers(PyObject* const* a, int n, double* out)
{
    for (int i = 0; i < n; ++i) {
        out[i] = PyFloat_AsDouble(a[i]);
        if (out[i] == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            return false;
        }
    }
    return true;
}

bool same_shapes(const std::vector<const at::Tensor*>& a, const std::vector<const at::Tensor*>& b)
{
    for (size_t i = 0; i < a.size(); ++i)
        if (a[i]->sizes() != b[i]->sizes()) return false;
    return true;
}

// (matrices, steps, a, b, c, eps) -> list of their orthogonalised forms, or None
PyObject* orthogonalise(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    std::vector<const at::Tensor*> g;
    List l;
    double v[4];
    int steps;
    if (n != 6 || !integer(args[1], &steps) || !numbers(args + 2, 4, v) || !begin_list(args[0], &g, &l)) Py_RETURN_NONE;
    std::vector<at::Tensor> out;
    std::vector<void*> to;
    for (const at::Tensor* t : g) {
        out.push_back(at::empty_like(*t));
        to.push_back(out.back().data_ptr());
    }
    const scc_orthogonal_options o = {0.f, 0.f, 0.f, 0, steps, (float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    const scc_dtype dtype = g[0]->scalar_type() == at::kFloat ? SCC_F32 : SCC_BF16;
    const int rc = launch(l.ws, [&](void* st) {
        return scc_orthogonalise((int)g.size(), l.address.data(), to.data(), l.rows.data(), l.cols.data(), &o, dtype, l.ws.data_ptr(),
                                 l.need, st);
    });
    if (rc != SCC_OK) Py_RETURN_NONE;
    PyObject* r = PyList_New((Py_ssize_t)out.size());
    for (size_t i = 0; r && i < out.size(); ++i) PyList_SET_ITEM(r, (Py_ssize_t)i, THPVariable_Wrap(out[i]));
    return r;
    END_HANDLE_TH_ERRORS
}

// Whether memory of a weight or a momentum belongs to another tensor of a step as well: its workgroups would write it at the same time.
bool overlap(std::initializer_list<const std::vector<const at::Tensor*>*> written, const std::vector<const at::Tensor*>& read)
{
    struct Span {
        uintptr_t first, last;
        bool written;
    };
    std::vector<Span> spans;
    auto add = [&](const std::vector<const at::Tensor*>& ts, bool w) {
        for (const at::Tensor* t : ts) spans.push_back({(uintptr_t)t->data_ptr(), (uintptr_t)t->data_ptr() + t->nbytes(), w});
    };
    for (const auto* ts : written) add(*ts, true);
    add(read, false);
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.first < b.first; });
    uintptr_t end = 0, end_written = 0;
    for (const Span& s : spans) {
        if (s.first < (s.written ? end : end_written)) return true;
        end = std::max(end, s.last);
        if (s.written) end_written = std::max(end_written, s.last);
    }
    return false;
}

// Tells autograd that a tensor has other values now, so that a graph which saved it is not run on them.
void moved(const std::vector<const at::Tensor*>& ts)
{
    for (const at::Tensor* t : ts)
        if (!t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// (weights, grads, momenta, lr, momentum, weight_decay, nesterov, steps, a, b, c, eps) -> the library's status, or None where the call is not
// plain.  It moves the caller's tensors, some of a list's even where a later launch fails, so a call that was made is not for scc.py to
// make again.
PyObject* orthogonal_step(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    std::vector<const at::Tensor*> w, g, m;
    List l;
    double v[3], e[4];
    int steps;
    if (n != 12 || !numbers(args + 3, 3, v) || !PyBool_Check(args[6]) || !integer(args[7], &steps) || !numbers(args + 8, 4, e) ||
        !begin_list(args[0], &w, &l))
        Py_RETURN_NONE;
    const Py_ssize_t count = (Py_ssize_t)w.size();
    if (!matrices(args[1], count, w[0]->scalar_type(), &g) || !matrices(args[2], count, at::kFloat, &m) || !same_shapes(w, g) ||
        !same_shapes(w, m) || overlap({&w, &m}, g))
        Py_RETURN_NONE;
    std::vector<void*> from;
    std::vector<float*> momenta;
    for (Py_ssize_t i = 0; i < count; ++i) {
        from.push_back(g[i]->data_ptr());
        momenta.push_back((float*)m[i]->data_ptr());
    }
    const scc_orthogonal_options o = {(float)v[0], (float)v[1], (float)v[2], args[6] == Py_True, steps,
                                      (float)e[0], (float)e[1], (float)e[2], (float)e[3]};
    const scc_dtype dtype = w[0]->scalar_type() == at::kFloat ? SCC_F32 : SCC_BF16;
    const int rc = launch(l.ws, [&](void* st) {
        return scc_orthogonal_step((int)count, l.address.data(), from.data(), momenta.data(), l.rows.data(), l.cols.data(), &o, dtype,
                                   l.ws.data_ptr(), l.need, st);
    });
    if (rc == SCC_OK || rc == SCC_ERR_LAUNCH) {
        moved(w);
        moved(m);
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// ---- residual norm ----

// Gradients of a norm or a vocabulary loss under create_graph, as a function of all that they were computed from (x again for what there is not)
struct FirstOrderOf : torch::autograd::Function<FirstOrderOf> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext*, const at::Tensor& dx, const at::Tensor& dw,
                                                  const at::Tensor&, const at::Tensor&, const at::Tensor&, const at::Tensor&, const at::Tensor&)
    {
        return {dx.detach(), dw.detach()};
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext*, torch::autograd::variable_list)
    {
        TORCH_CHECK(false, "this operator has no second derivative");
    }
};

// f(a, b, c, ...) of scc.py, for what is not plain in a backward pass; the interpreter's lock is not held
template <typename F>
std::vector<at::Tensor> from_python(const char* name, F&& arguments)
{
    struct Locked {
        PyGILState_STATE s = PyGILState_Ensure();
        ~Locked() { PyGILState_Release(s); }
    } locked;
    std::vector<at::Tensor> g;
    PyObject* m = PyImport_ImportModule("paper_2101_00745_amd.scc");
    PyObject* f = m ? PyObject_GetAttrString(m, name) : nullptr;
    PyObject* a = f ? arguments() : nullptr;
    PyObject* r = a ? PyObject_CallObject(f, a) : nullptr;
    for (int i = 0; r && i < 2; ++i) g.push_back(THPVariable_Unpack(PyTuple_GetItem(r, i)));
    Py_XDECREF(r);
    Py_XDECREF(a);
    Py_XDECREF(f);
    Py_XDECREF(m);
    if (g.empty()) {
        python_error e;
        e.persist();
        throw e;
    }
    return g;
}

PyObject* wrapped(const at::Tensor& t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

bool no_modes() { return !c10::impl::TorchDispatchModeTLS::any_modes_set() && at::impl::PythonTorchFunctionTLS::stack_len() == 0; }

bool wants_gradient(const at::Tensor& t) { return t.requires_grad() && !t.is_inference() && !t._fw_grad(0).defined(); }

struct Map {
    int N, C, H, W;
    scc_dtype dtype;
};

// residual: undefined where there is none
bool norm_map(const at::Tensor& x, const at::Tensor& w, const at::Tensor& residual, Map* m)
{
    if (!plain(x) || !plain(w, x) || x.dim() != 4 || w.dim() != 1 || !fits(x) || w.size(0) != x.size(1)) return false;
    if (residual.defined() && (!plain(residual, x) || residual.sizes() != x.sizes())) return false;
    *m = {(int)x.size(0), (int)x.size(1), (int)x.size(2), (int)x.size(3), x.scalar_type() == at::kFloat ? SCC_F32 : SCC_BF16};
    return true;
}

struct NormCall {
    const at::Tensor *x, *w;
    at::Tensor residual;
    float eps;
    Map m;
};

// (x, w, residual or None, eps)
bool norm_call(PyObject* const* a, Py_ssize_t n, NormCall* c)
{
    if (n != 4 || !no_modes() || !THPVariable_CheckExact(a[0]) || !THPVariable_CheckExact(a[1]) || !PyFloat_CheckExact(a[3])) return false;
    c->x = &THPVariable_Unpack(a[0]);
    c->w = &THPVariable_Unpack(a[1]);
    if (a[2] != Py_None) {
        if (!THPVariable_CheckExact(a[2])) return false;
        c->residual = THPVariable_Unpack(a[2]);
    }
    c->eps = (float)PyFloat_AS_DOUBLE(a[3]);
    return norm_map(*c->x, *c->w, c->residual, &c->m);
}

// y and h (undefined without a residual); none where the call failed
std::vector<at::Tensor> norm_forward_of(const at::Tensor& x, const at::Tensor& w, const at::Tensor& residual, float eps, const Map& m)
{
    at::Tensor y = at::empty(x.sizes(), x.options()), h = residual.defined() ? at::empty(x.sizes(), x.options()) : at::Tensor();
    const int rc = launch(x, [&](void* st) {
        return scc_norm_forward(x.data_ptr(), address(residual), w.data_ptr(), address(h), y.data_ptr(), m.N, m.C, m.H, m.W, eps, m.dtype, st);
    });
    if (rc != SCC_OK) return {};
    return {y, h};
}

PyObject* norm_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    NormCall c;
    if (!norm_call(args, n, &c)) Py_RETURN_NONE;
    const std::vector<at::Tensor> o = norm_forward_of(*c.x, *c.w, c.residual, c.eps, c.m);
    if (o.empty()) Py_RETURN_NONE;
    return tuple_of({o[0], o[1].defined() ? o[1] : *c.x});
    END_HANDLE_TH_ERRORS
}

PyObject* norm_quantised(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    NormCall c;
    if (!norm_call(args, n, &c)) Py_RETURN_NONE;
    const at::Tensor &x = *c.x, &r = c.residual;
    at::Tensor q = at::empty(x.sizes(), x.options().dtype(at::kFloat8_e4m3fn));
    at::Tensor scale = at::empty({c.m.N, c.m.H, c.m.W}, x.options().dtype(at::kFloat));
    at::Tensor h = r.defined() ? at::empty(x.sizes(), x.options()) : at::Tensor();
    const int rc = launch(x, [&](void* st) {
        return scc_norm_quantised(x.data_ptr(), address(r), c.w->data_ptr(), address(h), (uint8_t*)q.data_ptr(), (float*)scale.data_ptr(), c.m.N,
                                  c.m.C, c.m.H, c.m.W, c.eps, c.m.dtype, st);
    });
    if (rc != SCC_OK) Py_RETURN_NONE;
    return tuple_of({q, scale, h.defined() ? h : x});
    END_HANDLE_TH_ERRORS
}

// nn.ResidualNormFunction for a plain call all of whose tensors want gradients
struct Norm {
    struct Refused {};

    static std::vector<at::Tensor> gradients(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& w, const at::Tensor& dy_,
                                             const at::Tensor& dh_, double eps)
    {
        const at::Tensor dy = dy_.defined() ? dy_.contiguous() : at::zeros_like(x), dh = dh_.defined() ? dh_.contiguous() : dh_;
        Map m;
        std::vector<at::Tensor> g;
        auto like = [&](const at::Tensor& t) { return plain(t, x) && t.sizes() == x.sizes(); };
        if (norm_map(x, w, residual, &m) && like(dy) && (!dh.defined() || like(dh))) {
            at::Tensor dx = at::empty_like(x), dw = at::empty_like(w);
            const size_t need = scc_norm_backward_workspace_bytes(m.N, m.C, m.H, m.W, m.dtype);
            const at::Tensor ws = scratch(need, x);
            const int rc = scc_norm_backward(x.data_ptr(), address(residual), w.data_ptr(), dy.data_ptr(), address(dh), dx.data_ptr(),
                                             dw.data_ptr(), m.N, m.C, m.H, m.W, (float)eps, m.dtype, m.dtype, address(ws), need, stream_of(x));
            if (rc == SCC_OK) g = {dx, dw};
        }
        if (g.empty())
            g = from_python("_norm_backward", [&]() {
                return Py_BuildValue("(NNNNNdO)", wrapped(x), wrapped(w), wrapped(dy), wrapped(residual), wrapped(dh), eps, Py_True);
            });
        if (at::GradMode::is_enabled())
            g = FirstOrderOf::apply(g[0], g[1], x, residual.defined() ? residual : x, w, dy, dh.defined() ? dh : dy);
        return g;
    }

    struct Plain : torch::autograd::Function<Plain> {
        static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w, double eps)
        {
            Map m;
            std::vector<at::Tensor> o;
            if (norm_map(x, w, at::Tensor(), &m)) o = norm_forward_of(x, w, at::Tensor(), (float)eps, m);
            if (o.empty()) throw Refused();
            ctx->save_for_backward({x, w});
            ctx->saved_data["eps"] = eps;
            ctx->set_materialize_grads(false);
            return o[0];
        }

        static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
        {
            if (!grads[0].defined()) return {at::Tensor(), at::Tensor(), at::Tensor()};
            const torch::autograd::variable_list s = ctx->get_saved_variables();
            const std::vector<at::Tensor> g = gradients(s[0], at::Tensor(), s[1], grads[0], at::Tensor(), ctx->saved_data["eps"].toDouble());
            return {g[0], g[1], at::Tensor()};
        }
    };

    struct Residual : torch::autograd::Function<Residual> {
        static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w,
                                                      const at::Tensor& residual, double eps)
        {
            Map m;
            std::vector<at::Tensor> o;
            if (norm_map(x, w, residual, &m)) o = norm_forward_of(x, w, residual, (float)eps, m);
            if (o.empty()) throw Refused();
            // in binary32 the sum stands for both; in bf16 it is rounded
            if (m.dtype == SCC_F32) ctx->save_for_backward({w, o[1]});
            else ctx->save_for_backward({w, x, residual});
            ctx->saved_data["eps"] = eps;
            ctx->set_materialize_grads(false);
            return {o[0], o[1]};
        }

        static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
        {
            if (!grads[0].defined() && !grads[1].defined()) return {at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
            const torch::autograd::variable_list s = ctx->get_saved_variables();
            const std::vector<at::Tensor> g = gradients(s[1], s.size() > 2 ? s[2] : at::Tensor(), s[0], grads[0], grads[1],
                                                        ctx->saved_data["eps"].toDouble());
            return {g[0], g[1], g[0], at::Tensor()};
        }
    };
};

PyObject* norm_block(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    NormCall c;
    if (!at::GradMode::is_enabled() || !norm_call(args, n, &c) || !wants_gradient(*c.x) || !wants_gradient(*c.w) ||
        (c.residual.defined() && !wants_gradient(c.residual)))
        Py_RETURN_NONE;
    try {
        if (!c.residual.defined()) return tuple_of({Norm::Plain::apply(*c.x, *c.w, (double)c.eps), *c.x});
        const torch::autograd::variable_list o = Norm::Residual::apply(*c.x, *c.w, c.residual, (double)c.eps);
        return tuple_of({o[0], o[1]});
    } catch (const Norm::Refused&) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}

// ---- vocabulary loss ----

struct LossCall {
    const at::Tensor *x, *w, *target;
    int code;
    long long ignored;
    Map m;
    int V;
};

bool loss_map(const at::Tensor& x, const at::Tensor& w, const at::Tensor& target, Map* m, int* V)
{
    if (!plain(x) || !plain(w, x) || x.dim() != 4 || w.dim() != 2 || !fits(x) || !fits(w) || w.size(1) != x.size(1)) return false;
    if (!target.defined() || !target.is_cuda() || target.scalar_type() != at::kLong || !target.is_contiguous() || target.dim() != 3 ||
        target.get_device() != x.get_device() || target.size(0) != x.size(0) || target.size(1) != x.size(2) || target.size(2) != x.size(3))
        return false;
    *m = {(int)x.size(0), (int)x.size(1), (int)x.size(2), (int)x.size(3), x.scalar_type() == at::kFloat ? SCC_F32 : SCC_BF16};
    *V = (int)w.size(0);
    return true;
}

// (x, w, target, code, ignored)
bool loss_call(PyObject* const* a, Py_ssize_t n, LossCall* c)
{
    if (n != 5 || !no_modes() || !PyLong_CheckExact(a[3]) || !PyLong_CheckExact(a[4])) return false;
    for (int i = 0; i < 3; ++i)
        if (!THPVariable_CheckExact(a[i])) return false;
    c->x = &THPVariable_Unpack(a[0]);
    c->w = &THPVariable_Unpack(a[1]);
    c->target = &THPVariable_Unpack(a[2]);
    int overflow = 0, more = 0;
    c->code = (int)PyLong_AsLongAndOverflow(a[3], &overflow);
    c->ignored = PyLong_AsLongLongAndOverflow(a[4], &more);
    return !overflow && !more && loss_map(*c->x, *c->w, *c->target, &c->m, &c->V);
}

// loss and lse; none where the call failed
std::vector<at::Tensor> loss_of(const at::Tensor& x, const at::Tensor& w, const at::Tensor& target, int code, long long ignored, const Map& m, int V)
{
    const at::TensorOptions f = x.options().dtype(at::kFloat);
    at::Tensor lse = at::empty(target.sizes(), f), loss = code == SCC_NONE ? at::empty(target.sizes(), f) : at::empty({}, f);
    const size_t need = scc_vocabulary_loss_workspace_bytes(m.N, m.C, m.H, m.W, V, (scc_reduction)code, m.dtype);
    const at::Tensor ws = scratch(need, x);
    const int rc = launch(x, [&](void* st) {
        return scc_vocabulary_loss(x.data_ptr(), w.data_ptr(), (const long long*)target.data_ptr(), (float*)loss.data_ptr(), (float*)lse.data_ptr(),
                                   m.N, m.C, m.H, m.W, V, ignored, (scc_reduction)code, m.dtype, address(ws), need, st);
    });
    if (rc != SCC_OK) return {};
    return {loss, lse};
}

PyObject* vocabulary_loss(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    LossCall c;
    if (!loss_call(args, n, &c)) Py_RETURN_NONE;
    const std::vector<at::Tensor> o = loss_of(*c.x, *c.w, *c.target, c.code, c.ignored, c.m, c.V);
    if (o.empty()) Py_RETURN_NONE;
    return tuple_of({o[0], o[1]});
    END_HANDLE_TH_ERRORS
}

// nn.VocabularyLossFunction for a plain call whose x and weight want gradients
struct Loss : torch::autograd::Function<Loss> {
    struct Refused {};

    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w, const at::Tensor& target, int64_t code,
                              int64_t ignored)
    {
        Map m;
        int V;
        std::vector<at::Tensor> o;
        if (loss_map(x, w, target, &m, &V)) o = loss_of(x, w, target, (int)code, ignored, m, V);
        if (o.empty()) throw Refused();
        ctx->save_for_backward({x, w, target, o[1]});
        ctx->saved_data["code"] = code;
        ctx->saved_data["ignored"] = ignored;
        return o[0];
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const torch::autograd::variable_list s = ctx->get_saved_variables();
        const at::Tensor &x = s[0], &w = s[1], &target = s[2], &lse = s[3];
        const at::Tensor d = grads[0].contiguous();
        const int64_t code = ctx->saved_data["code"].toInt(), ignored = ctx->saved_data["ignored"].toInt();
        Map m;
        int V;
        std::vector<at::Tensor> g;
        auto like = [&](const at::Tensor& t, const at::Tensor& of) { return plain(t) && t.scalar_type() == at::kFloat && t.sizes() == of.sizes(); };
        if (loss_map(x, w, target, &m, &V) && like(lse, target) && (code == SCC_NONE ? like(d, target) : plain(d) && d.scalar_type() == at::kFloat && d.dim() == 0)) {
            at::Tensor dx = at::empty_like(x), dw = at::empty_like(w);
            const size_t need = scc_vocabulary_gradients_workspace_bytes(m.N, m.C, m.H, m.W, V, m.dtype);
            const at::Tensor ws = scratch(need, x);
            const int rc = scc_vocabulary_gradients(x.data_ptr(), w.data_ptr(), (const long long*)target.data_ptr(), (const float*)lse.data_ptr(),
                                                    (const float*)d.data_ptr(), dx.data_ptr(), dw.data_ptr(), m.N, m.C, m.H, m.W, V, ignored,
                                                    (scc_reduction)code, m.dtype, m.dtype, address(ws), need, stream_of(x));
            if (rc == SCC_OK) g = {dx, dw};
        }
        if (g.empty())
            g = from_python("_vocabulary_gradients", [&]() {
                return Py_BuildValue("(NNNNNLLO)", wrapped(x), wrapped(w), wrapped(target), wrapped(lse), wrapped(d), (long long)code,
                                     (long long)ignored, Py_True);
            });
        if (at::GradMode::is_enabled()) g = FirstOrderOf::apply(g[0], g[1], x, w, d, x, w);
        return {g[0], g[1], at::Tensor(), at::Tensor(), at::Tensor()};
    }
};

PyObject* vocabulary_block(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    LossCall c;
    if (!at::GradMode::is_enabled() || !loss_call(args, n, &c) || !wants_gradient(*c.x) || !wants_gradient(*c.w)) Py_RETURN_NONE;
    try {
        return THPVariable_Wrap(Loss::apply(*c.x, *c.w, *c.target, (int64_t)c.code, (int64_t)c.ignored));
    } catch (const Loss::Refused&) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}

// ---- AdamW ----

// A list of dense tensors of one type on the current device
bool tensors(PyObject* o, Py_ssize_t count, at::ScalarType type, std::vector<const at::Tensor*>* out)
{
    if (!PyList_CheckExact(o) || PyList_GET_SIZE(o) != count) return false;
    out->reserve(count);
    for (Py_ssize_t i = 0; i < count; ++i) {
        PyObject* e = PyList_GET_ITEM(o, i);
        if (!THPVariable_CheckExact(e)) return false;
        const at::Tensor& t = THPVariable_Unpack(e);
        if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || !t.is_contiguous() || t.scalar_type() != type ||
            t.numel() < 1 || t.get_device() != c10::hip::current_device())
            return false;
        out->push_back(&t);
    }
    return true;
}

// What a step works on: weights, gradients, states and, in 8 bits, their scales
struct AdamwLists {
    std::vector<const at::Tensor*> l[6];
    at::ScalarType type;
    bool bytes;
};

// (weights, grads, first, second, first scales or None, second scales or None); false where they are not plain or do not fit together
bool adamw_lists(PyObject* const* args, AdamwLists* o)
{
    if (!no_modes() || !PyList_CheckExact(args[0]) || PyList_GET_SIZE(args[0]) < 1 || PyList_GET_SIZE(args[0]) > INT_MAX) return false;
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    PyObject* e = PyList_GET_ITEM(args[0], 0);
    if (!THPVariable_CheckExact(e)) return false;
    const at::ScalarType type = THPVariable_Unpack(e).scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) return false;
    const bool bytes = args[4] != Py_None;
    const at::ScalarType state = bytes ? at::kFloat8_e4m3fn : at::kFloat;
    std::vector<const at::Tensor*>(&l)[6] = o->l;
    if ((args[5] != Py_None) != bytes || !tensors(args[0], count, type, &l[0]) || !tensors(args[1], count, type, &l[1]) ||
        !tensors(args[2], count, state, &l[2]) || !tensors(args[3], count, state, &l[3]) ||
        (bytes && (!tensors(args[4], count, at::kFloat, &l[4]) || !tensors(args[5], count, at::kFloat, &l[5]))))
        return false;
    if (!same_shapes(l[0], l[1]) || !same_shapes(l[0], l[2]) || !same_shapes(l[0], l[3])) return false;
    for (Py_ssize_t j = 0; bytes && j < count; ++j) {
        const int64_t blocks = (l[0][j]->numel() + 255) / 256;
        if (l[4][j]->numel() != blocks || l[5][j]->numel() != blocks) return false;
    }
    o->type = type;
    o->bytes = bytes;
    return !overlap({&l[0], &l[2], &l[3], &l[4], &l[5]}, l[1]);
}

// The same arguments -> True where a step on them is made here, or None
PyObject* adamw_fits(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    AdamwLists a;
    if (n != 6 || !adamw_lists(args, &a)) Py_RETURN_NONE;
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// (weights, grads, first, second, first scales or None, second scales or None, lr, step, b1, b2, eps, weight_decay, seed) -> the library's status, or
// None where the call is not plain; as orthogonal_step
PyObject* adamw_step(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    double v[5];
    AdamwLists a;
    if (n != 13 || !PyLong_CheckExact(args[7]) || !PyLong_CheckExact(args[12]) || !numbers(args + 6, 1, v) || !numbers(args + 8, 4, v + 1) ||
        !adamw_lists(args, &a))
        Py_RETURN_NONE;
    const size_t count = a.l[0].size();
    std::vector<long long> sizes(count);
    std::vector<void*> at[6];
    for (int i = 0; i < (a.bytes ? 6 : 4); ++i) {
        at[i].resize(count);
        for (size_t j = 0; j < count; ++j) at[i][j] = a.l[i][j]->data_ptr();
    }
    for (size_t j = 0; j < count; ++j) sizes[j] = a.l[0][j]->numel();
    int overflow = 0;
    const long long step = PyLong_AsLongLongAndOverflow(args[7], &overflow);
    if (overflow) Py_RETURN_NONE;
    const scc_adamw_options o = {v[0], v[1], v[2], v[3], v[4], (uint64_t)PyLong_AsUnsignedLongLongMask(args[12])};
    const int rc = launch(*a.l[0][0], [&](void* st) {
        return scc_adamw_step((int)count, at[0].data(), at[1].data(), at[2].data(), at[3].data(), a.bytes ? (float* const*)at[4].data() : nullptr,
                              a.bytes ? (float* const*)at[5].data() : nullptr, sizes.data(), &o, step, nullptr, a.type == at::kFloat ? SCC_F32 : SCC_BF16, st);
    });
    if (rc == SCC_OK || rc == SCC_ERR_LAUNCH)
        for (int i = 0; i < 6; ++i)
            if (i != 1) moved(a.l[i]);
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

#define METHOD(name, doc) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, doc}
PyMethodDef methods[] = {METHOD(forward, "(x, w, cg, co) -> y or None"), METHOD(backward, "(x, dy, w, cg, co) -> (dx, dw) or None"),
                         METHOD(dw_forward, "(x, kdw, w, cg, co, stride) -> y or None"),
                         METHOD(dw_block, "(x, kdw, w, cg, co, stride) -> y under autograd, or None"),
                         METHOD(dw_backward, "(x, kdw, w, dy, cg, co, stride, stored) -> (dx, dkdw, dw) or None"),
                         METHOD(gated_forward, "(x, w, cg, co, act) -> y or None"),
                         METHOD(gated_backward, "(x, w, dy, cg, co, act, stored) -> (dx, dw) or None"),
                         METHOD(gated_block, "(x, w, cg, co, act) -> y under autograd, or None"),
                         METHOD(orthogonalise, "(matrices, steps, a, b, c, eps) -> list or None"),
                         METHOD(orthogonal_step, "(weights, grads, momenta, lr, momentum, weight_decay, nesterov, steps, a, b, c, eps) -> status or None"),
                         METHOD(norm_forward, "(x, w, residual or None, eps) -> (y, h) or None"),
                         METHOD(norm_quantised, "(x, w, residual or None, eps) -> (q, scale, h) or None"),
                         METHOD(norm_block, "(x, w, residual or None, eps) -> (y, h) under autograd, or None"),
                         METHOD(vocabulary_loss, "(x, w, target, reduction, ignored) -> (loss, lse) or None"),
                         METHOD(vocabulary_block, "(x, w, target, reduction, ignored) -> loss under autograd, or None"),
                         METHOD(adamw_fits, "(weights, grads, first, second, first scales, second scales) -> True or None"),
                         METHOD(adamw_step, "(weights, grads, first, second, first scales, second scales, lr, step, b1, b2, eps, weight_decay, seed) -> status or None"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch (and interpreter) whose inlined types this code was compiled with; scc.py compares it before the first call
PyMODINIT_FUNC PyInit__binding()
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", SCC_BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
