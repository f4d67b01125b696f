// The Python binding's fast path: one call from Python checks the tensors of
// an entry point, takes a workspace where none is given, finds torch's
// current stream and calls libiabn.  Marshalling only, as in __init__.py,
// which this does not replace: whatever is not the plain case (a wrong
// argument, a tensor subclass, an explicit stream, tensors on another device
// than the current one) returns NotImplemented,
// and the Python function then does the same checks and reports what is
// wrong.
//
// Why native: the same checks in Python and a ctypes call of 17 arguments
// took 10-13 us per call, more than the kernels of a small layer.

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <cxxabi.h>
#include <torch/csrc/autograd/python_variable.h>

#include "iabn.h"

namespace {

// The entry points, in the order of the table that each call is given (the
// addresses in one loaded libiabn): see _NATIVE in __init__.py.
enum Op : long {
    kWorkspaceSize,
    kForwardTrain,
    kForwardTrainNoalloc,
    kForwardEval,
    kBackward,
    kBackwardII,
    kStdForward,
    kStdBackward,
    kCkptForward,
    kCkptRecompute,
    kCkptBackward,
    kOps,
    // The feed-forward sublayer's, each with a function of its own below.
    kDropout = kOps,
    kResnormForward,
    kResnormWorkspaceSize,
    kResnormBackward,
    kFfnWorkspaceSize,
    kFfnForward,
    kFfnBackward
};

// What follows the table and the op in a call: activation tensors,
// per-channel tensors, floats, then a workspace (or None) if it takes one.
struct Shape {
    int big, chan, floats;
    bool workspace;
};
constexpr Shape kShapes[kOps] = {{0, 0, 0, false}, {1, 6, 3, true},  {1, 6, 3, false}, {1, 4, 2, false},
                                 {2, 5, 2, true},  {2, 5, 2, true},  {2, 6, 3, true},  {3, 6, 2, true},
                                 {2, 6, 3, true},  {2, 2, 1, false}, {2, 5, 2, true}};

PyObject* not_plain() {
    PyErr_Clear();
    Py_RETURN_NOTIMPLEMENTED;
}

int dtype_code(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return IABN_F32;
        case at::kHalf: return IABN_F16;
        case at::kBFloat16: return IABN_BF16;
        default: return -1;
    }
}

// A launch on a default stream, which has no device of its own, goes to the
// thread's current one.
bool on_current(const at::Device& dev) { return c10::hip::current_device() == dev.index(); }

template <typename Fn>
Fn* entry(void* const* table, Op op) {
    return reinterpret_cast<Fn*>(table[op]);
}

// The call itself, without the GIL: takes a workspace (`own`) and launches.
int launch(void* const* table, Op op, int code, int64_t N, int64_t C, int64_t HW, void* const (&big)[3],
           float* const (&chan)[6], const float (&f)[3], at::Device dev, bool own, at::Tensor& ws) {
    if (own) {
        const size_t need =
            entry<decltype(iabn_workspace_size)>(table, kWorkspaceSize)(N, C, HW, code);
        ws = at::empty({static_cast<int64_t>(need ? need : 1)},
                       at::TensorOptions().dtype(at::kByte).device(dev));
    }
    void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? ws.numel() * ws.element_size() : 0;
    void* const st = c10::hip::getCurrentHIPStream(dev.index()).stream();
    switch (op) {
        case kForwardTrain:
            return entry<decltype(iabn_forward_train)>(table, op)(
                big[0], code, chan[0], chan[1], chan[2], chan[3], chan[4], chan[5], f[0], f[1], f[2], N,
                C, HW, wp, wb, st);
        case kForwardTrainNoalloc:
            return entry<decltype(iabn_forward_train_noalloc)>(table, op)(
                big[0], code, chan[0], chan[1], chan[2], chan[3], chan[4], chan[5], f[0], f[1], f[2], N,
                C, HW, st);
        case kForwardEval:
            return entry<decltype(iabn_forward_eval)>(table, op)(
                big[0], code, chan[0], chan[1], chan[2], chan[3], f[0], f[1], N, C, HW, st);
        case kBackward:
        case kBackwardII:
            return entry<decltype(iabn_backward)>(table, op)(
                big[0], big[1], code, chan[0], chan[1], chan[2], chan[3], chan[4], f[0], f[1], N, C, HW,
                wp, wb, st);
        case kStdForward:
            return entry<decltype(iabn_std_forward_train)>(table, op)(
                big[0], big[1], code, chan[0], chan[1], chan[2], chan[3], chan[4], chan[5], f[0], f[1],
                f[2], N, C, HW, wp, wb, st);
        case kStdBackward:
            return entry<decltype(iabn_std_backward)>(table, op)(
                big[0], big[1], big[2], code, chan[0], chan[1], chan[2], chan[3], chan[4], chan[5], f[0],
                f[1], N, C, HW, wp, wb, st);
        case kCkptForward:
            return entry<decltype(iabn_ckpt_forward_train)>(table, op)(
                big[0], big[1], code, chan[0], chan[1], chan[2], chan[3], chan[4], chan[5], f[0], f[1],
                f[2], N, C, HW, wp, wb, st);
        case kCkptRecompute:
            return entry<decltype(iabn_ckpt_recompute)>(table, op)(
                big[0], big[1], code, chan[0], chan[1], f[0], N, C, HW, st);
        default:
            return entry<decltype(iabn_ckpt_backward)>(table, op)(
                big[0], big[1], code, chan[0], chan[1], chan[2], chan[3], chan[4], f[0], f[1], N, C, HW,
                wp, wb, st);
    }
}

PyObject* call_checked(PyObject* const* args, Py_ssize_t n) {
    if (n < 2) return not_plain();
    void* const* table = static_cast<void* const*>(PyLong_AsVoidPtr(args[0]));
    const long opn = PyLong_AsLong(args[1]);
    if (table == nullptr || opn <= kWorkspaceSize || opn >= kOps) return not_plain();
    const Op op = static_cast<Op>(opn);
    const Shape& s = kShapes[op];
    if (n != 2 + s.big + s.chan + s.floats + (s.workspace ? 1 : 0)) return not_plain();
    args += 2;

    void* big[3];
    int64_t N = 0, C = 0, HW = 1;
    int code = -1;
    at::Device dev(at::kCPU);
    for (int i = 0; i < s.big; ++i) {
        if (!THPVariable_CheckExact(args[i])) return not_plain();
        const at::Tensor& t = THPVariable_Unpack(args[i]);
        if (t.dim() < 2 || !t.is_cuda() || !t.is_contiguous()) return not_plain();
        if (i == 0) {
            N = t.size(0);
            C = t.size(1);
            for (int64_t d = 2; d < t.dim(); ++d) HW *= t.size(d);
            code = dtype_code(t.scalar_type());
            dev = t.device();
            if (code < 0) return not_plain();
        } else {
            int64_t hw = 1;
            for (int64_t d = 2; d < t.dim(); ++d) hw *= t.size(d);
            if (t.size(0) != N || t.size(1) != C || hw != HW || dtype_code(t.scalar_type()) != code ||
                t.device() != dev)
                return not_plain();
        }
        big[i] = t.data_ptr();
    }
    args += s.big;
    float* chan[6];
    for (int i = 0; i < s.chan; ++i) {
        if (!THPVariable_CheckExact(args[i])) return not_plain();
        const at::Tensor& t = THPVariable_Unpack(args[i]);
        if (t.scalar_type() != at::kFloat || !t.is_contiguous() || t.numel() != C || t.device() != dev)
            return not_plain();
        chan[i] = static_cast<float*>(t.data_ptr());
    }
    args += s.chan;
    float f[3];
    for (int i = 0; i < s.floats; ++i) {
        const double v = PyFloat_Check(args[i]) || PyLong_Check(args[i]) ? PyFloat_AsDouble(args[i]) : -1.0;
        if (PyErr_Occurred() || !(PyFloat_Check(args[i]) || PyLong_Check(args[i]))) return not_plain();
        f[i] = static_cast<float>(v);
    }
    args += s.floats;
    at::Tensor ws;
    bool own = false;
    if (s.workspace) {
        own = args[0] == Py_None;
        if (!own) {
            if (!THPVariable_CheckExact(args[0])) return not_plain();
            ws = THPVariable_Unpack(args[0]);
            if (ws.device() != dev || !ws.is_contiguous()) return not_plain();
        }
    }

    if (!on_current(dev)) return not_plain();

    // An allocation can wait for the device and a launch for room in the
    // queue, so other Python threads go on meanwhile.
    int rc = 0;
    PyThreadState* thread = PyEval_SaveThread();
    try {
        rc = launch(table, op, code, N, C, HW, big, chan, f, dev, own, ws);
    } catch (...) {
        PyEval_RestoreThread(thread);
        throw;
    }
    PyEval_RestoreThread(thread);
    return PyLong_FromLong(rc);
}

// call(table, op, tensors..., floats...[, workspace]) -> status, or
// NotImplemented (nothing was done).  A C++ exception before the launch (no
// memory for a workspace, a tensor without storage) is left to the Python
// path to meet again and report.
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        return call_checked(args, n);
    } catch (abi::__forced_unwind&) {
        throw;  // the interpreter ends this thread
    } catch (...) {
        return not_plain();
    }
}

// ---------------------------------------------------------------- the sublayer

// The arguments of a sublayer's call, taken one after the other; `plain` turns
// false at the first one that is not as it should be.
struct Args {
    PyObject* const* at;
    bool plain = true;
    int64_t R = -1, C = 0;
    int code = -1;
    at::Device dev{at::kCPU};

    const at::Tensor* tensor(bool optional) {
        PyObject* const o = *at++;
        if (optional && o == Py_None) return nullptr;
        if (!plain || !THPVariable_CheckExact(o)) {
            plain = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) plain = false;
        return plain ? &t : nullptr;
    }
    // A tensor of [..., C]: the first one of the call says which R and C.
    void* rows(bool optional = false) {
        const at::Tensor* const t = tensor(optional);
        if (t == nullptr) return nullptr;
        const int64_t d = t->dim();
        if (d < 1) return plain = false, nullptr;
        if (R < 0) {
            C = t->size(d - 1);
            R = 1;
            for (int64_t i = 0; i + 1 < d; ++i) R *= t->size(i);
            code = dtype_code(t->scalar_type());
            dev = t->device();
            if (code < 0) plain = false;
        } else if (t->size(d - 1) != C || t->numel() != R * C || dtype_code(t->scalar_type()) != code ||
                   t->device() != dev) {
            plain = false;
        }
        return plain ? t->data_ptr() : nullptr;
    }
    // A tensor of the rows' type, of whole rows of C; their number in `n`.
    void* gate(int64_t& n) {
        n = 0;
        const at::Tensor* const t = tensor(true);
        if (t == nullptr) return nullptr;
        if (t->dim() < 1 || t->size(t->dim() - 1) != C || C == 0 || dtype_code(t->scalar_type()) != code ||
            t->device() != dev)
            return plain = false, nullptr;
        n = t->numel() / C;
        return t->data_ptr();
    }
    // A tensor of the rows' type and `n` values whose last dim is `last`.
    void* matrix(int64_t n, int64_t last, bool optional = false) {
        const at::Tensor* const t = tensor(optional);
        if (t == nullptr) return nullptr;
        if (t->dim() < 1 || t->size(t->dim() - 1) != last || t->numel() != n ||
            dtype_code(t->scalar_type()) != code || t->device() != dev)
            return plain = false, nullptr;
        return t->data_ptr();
    }
    // A weight, [F, C]; the first one of the call says which F.
    int64_t F = 0;
    void* first_weight() {
        const at::Tensor* const t = tensor(false);
        if (t == nullptr) return nullptr;
        if (t->dim() != 2 || t->size(1) != C || dtype_code(t->scalar_type()) != code || t->device() != dev)
            return plain = false, nullptr;
        F = t->size(0);
        return t->data_ptr();
    }
    float* floats(int64_t n) {
        const at::Tensor* const t = tensor(true);
        if (t == nullptr) return nullptr;
        if (t->scalar_type() != at::kFloat || t->numel() != n || t->device() != dev)
            return plain = false, nullptr;
        return static_cast<float*>(t->data_ptr());
    }
    float number() {
        PyObject* const o = *at++;
        if (!plain || !(PyFloat_Check(o) || PyLong_Check(o))) return plain = false, 0.0f;
        const double v = PyFloat_AsDouble(o);
        if (PyErr_Occurred()) plain = false;
        return static_cast<float>(v);
    }
    int choice() {
        PyObject* const o = *at++;
        if (!plain || !PyLong_CheckExact(o)) return plain = false, 0;
        const long v = PyLong_AsLong(o);
        if (PyErr_Occurred() || v < 0 || v > 1000) plain = false;
        return static_cast<int>(v);
    }
    uint64_t word() {
        PyObject* const o = *at++;
        if (!plain || !PyLong_CheckExact(o)) return plain = false, 0;
        const uint64_t v = PyLong_AsUnsignedLongLong(o);
        if (PyErr_Occurred()) plain = false;
        return v;
    }
    // The caller's workspace, or none (`own`).
    at::Tensor workspace(bool& own) {
        PyObject* const o = *at++;
        own = o == Py_None;
        if (own) return at::Tensor();
        if (!plain || !THPVariable_CheckExact(o)) return plain = false, at::Tensor();
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.device() != dev || !t.is_contiguous()) plain = false;
        return t;
    }
    bool ready() const { return plain && on_current(dev); }
    void* stream() const { return c10::hip::getCurrentHIPStream(dev.index()).stream(); }
    void take(at::Tensor& ws, bool own, size_t need) const {
        if (own)
            ws = at::empty({static_cast<int64_t>(need ? need : 1)},
                           at::TensorOptions().dtype(at::kByte).device(dev));
    }
};

size_t bytes_of(const at::Tensor& t) { return t.numel() * t.element_size(); }

// Runs `fn` without the GIL (an allocation can wait for the device and a
// launch for room in the queue).
template <typename Fn>
PyObject* without_gil(Fn fn) {
    int rc = 0;
    PyThreadState* thread = PyEval_SaveThread();
    try {
        rc = fn();
    } catch (...) {
        PyEval_RestoreThread(thread);
        throw;
    }
    PyEval_RestoreThread(thread);
    return PyLong_FromLong(rc);
}

PyObject* dropout_checked(void* const* table, Args& a) {
    void* const x = a.rows();
    void* const y = a.rows();
    const float p = a.number();
    const uint64_t seed = a.word(), offset = a.word();
    if (!a.ready()) return not_plain();
    return without_gil([&] {
        return entry<decltype(iabn_dropout)>(table, kDropout)(x, y, a.code, p, seed, offset, a.R, a.C,
                                                              a.stream());
    });
}

PyObject* resnorm_forward_checked(void* const* table, Args& a) {
    void* const x = a.rows();
    void* const h = a.rows(true);
    void* const r = a.rows(true);
    void* const u = a.rows(true);
    int64_t groups;
    void* const gate = a.gate(groups);
    const int post = a.choice();
    float* const post_w = a.floats(a.C);
    float* const post_b = a.floats(a.C);
    const int pre = a.choice();
    float* const pre_w = a.floats(a.C);
    float* const pre_b = a.floats(a.C);
    float* const post_stats = a.floats(2 * a.R);
    float* const pre_stats = a.floats(2 * a.R);
    const float alpha = a.number(), beta = a.number(), eps = a.number(), p = a.number();
    const uint64_t seed = a.word(), offset = a.word();
    if (!a.ready()) return not_plain();
    return without_gil([&] {
        return entry<decltype(iabn_resnorm_forward)>(table, kResnormForward)(
            x, h, r, u, a.code, gate, groups, post, post_w, post_b, pre, pre_w, pre_b, post_stats,
            pre_stats, alpha, beta, eps, p, seed, offset, a.R, a.C, a.stream());
    });
}

PyObject* resnorm_backward_checked(void* const* table, Args& a) {
    void* const dr = a.rows(true);
    void* const du = a.rows(true);
    void* const r = a.rows(true);
    void* const h = a.rows(true);
    void* const dx = a.rows(true);
    void* const dh = a.rows(true);
    if (a.R < 0) return not_plain();
    int64_t groups, dgroups;
    void* const gate = a.gate(groups);
    const int post = a.choice();
    float* const post_w = a.floats(a.C);
    float* const post_b = a.floats(a.C);
    const int pre = a.choice();
    float* const pre_w = a.floats(a.C);
    float* const post_stats = a.floats(2 * a.R);
    float* const pre_stats = a.floats(2 * a.R);
    void* const dgate = a.gate(dgroups);
    float* const dpost_w = a.floats(a.C);
    float* const dpost_b = a.floats(a.C);
    float* const dpre_w = a.floats(a.C);
    float* const dpre_b = a.floats(a.C);
    const float alpha = a.number(), beta = a.number(), p = a.number();
    const uint64_t seed = a.word(), offset = a.word();
    bool own;
    at::Tensor ws = a.workspace(own);
    if (!a.ready() || (dgate && dgroups != groups)) return not_plain();
    return without_gil([&] {
        a.take(ws, own, entry<decltype(iabn_resnorm_workspace_size)>(table, kResnormWorkspaceSize)(
                            a.R, a.C, groups));
        return entry<decltype(iabn_resnorm_backward)>(table, kResnormBackward)(
            dr, du, r, h, dx, dh, a.code, gate, groups, post, post_w, post_b, pre, pre_w, post_stats,
            pre_stats, dgate, dpost_w, dpost_b, dpre_w, dpre_b, alpha, beta, p, seed, offset, a.R, a.C,
            ws.data_ptr(), bytes_of(ws), a.stream());
    });
}

PyObject* ffn_forward_checked(void* const* table, Args& a) {
    void* const x = a.rows();
    void* const wg = a.first_weight();
    void* const wu = a.matrix(a.F * a.C, a.C);
    void* const wd = a.matrix(a.C * a.F, a.F);
    void* const y = a.rows();
    void* const g = a.matrix(a.R * a.F, a.F, true);
    void* const u = a.matrix(a.R * a.F, a.F, true);
    const int act = a.choice();
    const float slope = a.number();
    bool own;
    at::Tensor ws = a.workspace(own);
    if (!a.ready()) return not_plain();
    return without_gil([&] {
        a.take(ws, own, entry<decltype(iabn_ffn_workspace_size)>(table, kFfnWorkspaceSize)(
                            a.R, a.C, a.F, a.code));
        return entry<decltype(iabn_ffn_forward)>(table, kFfnForward)(
            x, wg, wu, wd, y, g, u, a.code, act, slope, a.R, a.C, a.F, ws.data_ptr(), bytes_of(ws),
            a.stream());
    });
}

PyObject* ffn_backward_checked(void* const* table, Args& a) {
    void* const dy = a.rows();
    void* const x = a.rows();
    // F stands in the weights, which come after g and u.
    PyObject* const* const at_g = a.at;
    a.at += 2;
    void* const wg = a.first_weight();
    void* const wu = a.matrix(a.F * a.C, a.C);
    void* const wd = a.matrix(a.C * a.F, a.F);
    PyObject* const* const at_dx = a.at;
    a.at = at_g;
    void* const g = a.matrix(a.R * a.F, a.F);
    void* const u = a.matrix(a.R * a.F, a.F);
    a.at = at_dx;
    void* const dx = a.rows();
    void* const dg = a.matrix(a.R * a.F, a.F);
    void* const du = a.matrix(a.R * a.F, a.F);
    void* const dwg = a.matrix(a.F * a.C, a.C);
    void* const dwu = a.matrix(a.F * a.C, a.C);
    void* const dwd = a.matrix(a.C * a.F, a.F);
    const int act = a.choice();
    const float slope = a.number();
    bool own;
    at::Tensor ws = a.workspace(own);
    if (!a.ready()) return not_plain();
    return without_gil([&] {
        a.take(ws, own, entry<decltype(iabn_ffn_workspace_size)>(table, kFfnWorkspaceSize)(
                            a.R, a.C, a.F, a.code));
        return entry<decltype(iabn_ffn_backward)>(table, kFfnBackward)(
            dy, x, g, u, wg, wu, wd, dx, dg, du, dwg, dwu, dwd, a.code, act, slope, a.R, a.C, a.F,
            ws.data_ptr(), bytes_of(ws), a.stream());
    });
}

// fn(table, arguments...) -> status or NotImplemented, as `call`.
template <PyObject* (*FN)(void* const*, Args&), Py_ssize_t N>
PyObject* sublayer(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        if (n != N + 1) return not_plain();
        void* const* table = static_cast<void* const*>(PyLong_AsVoidPtr(args[0]));
        if (table == nullptr) return not_plain();
        Args a{args + 1};
        return FN(table, a);
    } catch (abi::__forced_unwind&) {
        throw;
    } catch (...) {
        return not_plain();
    }
}

template <PyObject* (*FN)(void* const*, Args&), Py_ssize_t N>
PyCFunction method() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(sublayer<FN, N>));
}

PyMethodDef methods[] = {
    {"dropout", method<dropout_checked, 5>(), METH_FASTCALL, "iabn_dropout, as call"},
    {"resnorm_forward", method<resnorm_forward_checked, 19>(), METH_FASTCALL,
     "iabn_resnorm_forward, as call"},
    {"resnorm_backward", method<resnorm_backward_checked, 25>(), METH_FASTCALL,
     "iabn_resnorm_backward, as call"},
    {"ffn_forward", method<ffn_forward_checked, 10>(), METH_FASTCALL, "iabn_ffn_forward, as call"},
    {"ffn_backward", method<ffn_backward_checked, 16>(), METH_FASTCALL, "iabn_ffn_backward, as call"},
    {"call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call)), METH_FASTCALL,
     "call(table, op, tensors..., floats...[, workspace]) -> status or NotImplemented"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods,
                      nullptr,               nullptr,    nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
