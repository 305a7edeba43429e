// The part of the Python binding that runs on every call, in native code: a call's tensors become device pointers, its
// outputs and scratch are allocated, and the C ABI (include/picospec.h) is entered, without the interpreter in between.
// A round trip through ctypes and torch's Python allocation costs two to three microseconds per tensor allocated and up to
// six per call, more than the kernels of a small call take.  Plain CPython functions; tensors are torch's own.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <algorithm>
#include <cmath>
#include <stdexcept>
#include <string>

#include "../../include/picospec.h"

namespace {

struct BadArgument : std::runtime_error { using std::runtime_error::runtime_error; };

// The arguments of one call, converted one by one; an argument of the wrong kind ends the call with a TypeError.
struct Args {
    PyObject* const* a;
    Py_ssize_t n, at = 0;
    PyObject* next() {
        if (at >= n) throw BadArgument("too few arguments");
        return a[at++];
    }
    void* ptr() {                              // tensor or None
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) throw BadArgument("a tensor or None is expected");
        return THPVariable_Unpack(o).data_ptr();
    }
    const at::Tensor& tensor() {
        PyObject* o = next();
        if (!THPVariable_Check(o)) throw BadArgument("a tensor is expected");
        return THPVariable_Unpack(o);
    }
    template <class T> T* ptr() { return static_cast<T*>(ptr()); }
    int64_t i64() {
        const long long v = PyLong_AsLongLong(next());
        if (v == -1 && PyErr_Occurred()) throw BadArgument("");
        return v;
    }
    int i32() { return (int)i64(); }
    float f32() {
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) throw BadArgument("");
        return (float)v;
    }
    void* stream() { return (void*)(intptr_t)i64(); }
    struct Buffer { void* p; size_t bytes; };
    Buffer buffer() {                          // workspace: tensor or None
        PyObject* o = next();
        if (o == Py_None) return {nullptr, 0};
        if (!THPVariable_Check(o)) throw BadArgument("a tensor or None is expected");
        const at::Tensor& t = THPVariable_Unpack(o);
        return {t.data_ptr(), (size_t)t.nbytes()};
    }
    void done() const { if (at != n) throw BadArgument("too many arguments"); }
};

// f(), a call of the library, without the interpreter's lock where this thread has it: a call that waits for room in its stream's queue must not stop other Python threads
// (the engine runs backward calls without it)
template <class F>
int in_library(F f) {
    if (!PyGILState_Check()) return f();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

// Runs `call(args)` - which converts its arguments and returns the C function with them bound - and returns its code.
template <class F>
PyObject* enter(PyObject* const* argv, Py_ssize_t n, F call) {
    HANDLE_TH_ERRORS
    try {
        Args a{argv, n};
        auto bound = call(a);
        a.done();
        return PyLong_FromLong(in_library(bound));
    } catch (const BadArgument& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject* n_compress(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto z = a.ptr(); auto dt = a.i32(); auto ld = a.i64(); auto rows = a.i32(), V = a.i32(); auto T = a.f32(); auto k = a.i32(); auto top_p = a.f32();
        auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto mass = a.ptr<float>(); auto lse = a.ptr<float>();
        auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_compress(z, dt, ld, rows, V, T, k, top_p, idx, prob, count, mass, lse, ws.p, ws.bytes, s); };
    });
}

PyObject* n_sample_draft(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto mass = a.ptr<float>();
        auto k = a.i32(), rows = a.i32(); auto uni = a.ptr<float>(); auto tok = a.ptr<int32_t>(); auto q = a.ptr<float>(); auto s = a.stream();
        return [=] { return picospec_sample_draft(idx, prob, count, mass, k, rows, uni, tok, q, s); };
    });
}

struct Records { const int32_t* idx; const float* prob; const int32_t* count; const float* mass; int k; };
Records records(Args& a) { auto i = a.ptr<int32_t>(); auto p = a.ptr<float>(); auto c = a.ptr<int32_t>(); auto m = a.ptr<float>(); return {i, p, c, m, a.i32()}; }
struct Verdict { int32_t* n; float *p, *q, *mx, *sm, *lse; uint32_t* fl; };
Verdict verdict(Args& a) {
    auto n = a.ptr<int32_t>(); auto p = a.ptr<float>(); auto q = a.ptr<float>(); auto mx = a.ptr<float>(); auto sm = a.ptr<float>(); auto lse = a.ptr<float>();
    return {n, p, q, mx, sm, lse, a.ptr<uint32_t>()};
}
struct Target { const void* z; int dt; int64_t ld; int V; float T; int B, N; const int32_t* off; };
Target target(Args& a) {
    auto z = a.ptr(); auto dt = a.i32(); auto ld = a.i64(); auto V = a.i32(); auto T = a.f32(); auto B = a.i32(), N = a.i32();
    return {z, dt, ld, V, T, B, N, a.ptr<int32_t>()};
}
struct Draw { int32_t* tok; float* mass; uint32_t* fl; };
Draw draw(Args& a) { auto t = a.ptr<int32_t>(); auto m = a.ptr<float>(); return {t, m, a.ptr<uint32_t>()}; }

PyObject* n_verify(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto t = target(a); auto tok = a.ptr<int32_t>(); auto q = records(a); auto renorm = a.i32(); auto qs = a.ptr<float>(); auto uni = a.ptr<float>();
        auto o = verdict(a); auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_verify(t.z, t.dt, t.ld, t.V, t.T, t.B, t.N, t.off, tok, q.idx, q.prob, q.count, q.mass, q.k, renorm, qs, uni,
                                            o.n, o.p, o.q, o.mx, o.sm, o.lse, o.fl, ws.p, ws.bytes, s); };
    });
}

PyObject* n_verify_range(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto t = target(a); auto tok = a.ptr<int32_t>(); auto q = records(a); auto renorm = a.i32(); auto qs = a.ptr<float>(); auto uni = a.ptr<float>();
        auto pb = a.ptr<int32_t>(); auto pe = a.ptr<int32_t>(); auto g = a.i32();
        auto o = verdict(a); auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_verify_range(t.z, t.dt, t.ld, t.V, t.T, t.B, t.N, t.off, tok, q.idx, q.prob, q.count, q.mass, q.k, renorm, qs, uni,
                                                  pb, pe, g, o.n, o.p, o.q, o.mx, o.sm, o.lse, o.fl, ws.p, ws.bytes, s); };
    });
}

PyObject* n_round(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto zd = a.ptr(), zt = a.ptr(); auto dt = a.i32(); auto ldd = a.i64(), ldt = a.i64(); auto V = a.i32(); auto T = a.f32(); auto B = a.i32(), N = a.i32();
        auto off = a.ptr<int32_t>(); auto tok = a.ptr<int32_t>(); auto k = a.i32(); auto top_p = a.f32(); auto renorm = a.i32(); auto uni = a.ptr<float>();
        auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto mass = a.ptr<float>(); auto lse = a.ptr<float>();
        auto o = verdict(a); auto d = draw(a); auto ws = a.buffer(), own = a.buffer(); auto s = a.stream();
        if (own.p) ws = own;                     // (scratch(..) brings one only where the caller's does not serve)
        return [=] { return picospec_round(zd, zt, dt, ldd, ldt, V, T, B, N, off, tok, k, top_p, renorm, uni, idx, prob, count, mass, lse,
                                           o.n, o.p, o.q, o.mx, o.sm, o.lse, o.fl, d.tok, d.mass, d.fl, ws.p, ws.bytes, s); };
    });
}

PyObject* n_verify_sample(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto t = target(a); auto tok = a.ptr<int32_t>(); auto q = records(a); auto renorm = a.i32(); auto uni = a.ptr<float>();
        auto o = verdict(a); auto d = draw(a); auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_verify_sample(t.z, t.dt, t.ld, t.V, t.T, t.B, t.N, t.off, tok, q.idx, q.prob, q.count, q.mass, q.k, renorm, uni,
                                                   o.n, o.p, o.q, o.mx, o.sm, o.lse, o.fl, d.tok, d.mass, d.fl, ws.p, ws.bytes, s); };
    });
}

PyObject* n_verify_sample_static(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto t = target(a); auto tok = a.ptr<int32_t>(); auto q = records(a); auto renorm = a.i32(); auto uni = a.ptr<float>();
        auto o = verdict(a); auto d = draw(a); auto s = a.stream();
        return [=] { return picospec_verify_sample_static(t.z, t.dt, t.ld, t.V, t.T, t.B, t.N, t.off, tok, q.idx, q.prob, q.count, q.mass, q.k, renorm, uni,
                                                          o.n, o.p, o.q, o.mx, o.sm, o.lse, o.fl, d.tok, d.mass, d.fl, s); };
    });
}

template <auto CALL>
PyObject* n_sample_residual(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto t = target(a); auto na = a.ptr<int32_t>(); auto mx = a.ptr<float>(); auto sm = a.ptr<float>(); auto q = records(a); auto renorm = a.i32();
        auto uni = a.ptr<float>(); auto d = draw(a); auto ws = a.buffer(); auto s = a.stream();
        return [=] { return CALL(t.z, t.dt, t.ld, t.V, t.T, t.B, t.N, t.off, na, mx, sm, q.idx, q.prob, q.count, q.mass, q.k, renorm, uni,
                                 d.tok, d.mass, d.fl, ws.p, ws.bytes, s); };
    });
}

PyObject* n_row_stats(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto z = a.ptr(); auto dt = a.i32(); auto ld = a.i64(); auto rows = a.i32(), V = a.i32(); auto T = a.f32();
        auto mx = a.ptr<float>(); auto sm = a.ptr<float>(); auto lse = a.ptr<float>(); auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_row_stats_ws(z, dt, ld, rows, V, T, mx, sm, lse, ws.p, ws.bytes, s); };
    });
}

PyObject* n_compress_rejected(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto t = target(a); auto na = a.ptr<int32_t>(); auto k = a.i32(); auto top_p = a.f32();
        auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto mass = a.ptr<float>(); auto lse = a.ptr<float>();
        auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_compress_rejected(t.z, t.dt, t.ld, t.V, t.T, t.B, t.N, t.off, na, k, top_p, idx, prob, count, mass, lse, ws.p, ws.bytes, s); };
    });
}

PyObject* n_resample_sparse(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto t = target(a); auto na = a.ptr<int32_t>(); auto mx = a.ptr<float>(); auto sm = a.ptr<float>(); auto q = records(a); auto renorm = a.i32();
        auto uni = a.ptr<float>(); auto d = draw(a); auto s = a.stream();
        return [=] { return picospec_resample_sparse(t.z, t.dt, t.ld, t.V, t.T, t.B, t.N, t.off, na, mx, sm, q.idx, q.prob, q.count, q.mass, q.k, renorm, uni,
                                                     d.tok, d.mass, d.fl, nullptr, 0, s); };
    });
}

PyObject* n_pack_downlink(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto B = a.i32(); auto off = a.ptr<int32_t>(); auto na = a.ptr<int32_t>(); auto tok = a.ptr<int32_t>(); auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>();
        auto count = a.ptr<int32_t>(); auto k = a.i32(), fmt = a.i32(); auto wire = a.ptr(); auto cap = a.i64(); auto nb = a.ptr<int64_t>(); auto st = a.ptr<uint32_t>(); auto s = a.stream();
        return [=] { return picospec_pack_downlink(B, off, na, tok, idx, prob, count, k, fmt, wire, cap, nb, st, s); };
    });
}

PyObject* n_unpack_downlink(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto wire = a.ptr(); auto bytes = a.i64(); auto B = a.i32(), k = a.i32(); auto na = a.ptr<int32_t>(); auto tok = a.ptr<int32_t>();
        auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto mass = a.ptr<float>(); auto st = a.ptr<uint32_t>(); auto s = a.stream();
        return [=] { return picospec_unpack_downlink(wire, bytes, B, k, na, tok, idx, prob, count, mass, st, s); };
    });
}

PyObject* n_pack_uplink(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto B = a.i32(), N = a.i32(); auto off = a.ptr<int32_t>(); auto tok = a.ptr<int32_t>(); auto q = a.ptr<float>(); auto fmt = a.i32();
        auto wire = a.ptr(); auto cap = a.i64(); auto nb = a.ptr<int64_t>(); auto s = a.stream();
        return [=] { return picospec_pack_uplink(B, N, off, tok, q, fmt, wire, cap, nb, s); };
    });
}

PyObject* n_unpack_uplink(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto wire = a.ptr(); auto bytes = a.i64(); auto B = a.i32(), nm = a.i32(); auto off = a.ptr<int32_t>(); auto tok = a.ptr<int32_t>(); auto q = a.ptr<float>();
        auto st = a.ptr<uint32_t>(); auto s = a.stream();
        return [=] { return picospec_unpack_uplink(wire, bytes, B, nm, off, tok, q, st, s); };
    });
}

PyObject* n_sample(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto z = a.ptr(); auto dt = a.i32(); auto ld = a.i64(); auto rows = a.i32(), V = a.i32(); auto T = a.f32(); auto k = a.i32(); auto p = a.f32(), mp = a.f32();
        auto Tr = a.ptr<float>(); auto kr = a.ptr<int32_t>(); auto pr = a.ptr<float>(); auto mr = a.ptr<float>(); auto u = a.ptr<float>();
        auto tok = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto lse = a.ptr<float>();
        auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_sample(z, dt, ld, rows, V, T, k, p, mp, Tr, kr, pr, mr, u, tok, prob, count, lse, ws.p, ws.bytes, s); };
    });
}

PyObject* n_distill(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto z = a.ptr(); auto dt = a.i32(); auto ld = a.i64(); auto rows = a.i32(), V = a.i32(); auto T = a.f32();
        auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto k = a.i32(), tail = a.i32();
        auto weight = a.ptr<float>(); auto loss = a.ptr<float>(); auto accept = a.ptr<float>(); auto stats = a.ptr<double>();
        auto grad = a.ptr(); auto ldg = a.i64(); auto ws = a.buffer(); auto s = a.stream();
        return [=] { return picospec_distill(z, dt, ld, rows, V, T, idx, prob, count, k, tail, weight, loss, accept, stats, grad, ldg, ws.p, ws.bytes, s); };
    });
}

PyObject* n_distill_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return enter(v, n, [](Args& a) {
        auto z = a.ptr(); auto dt = a.i32(); auto ld = a.i64(); auto rows = a.i32(), V = a.i32(); auto T = a.f32();
        auto idx = a.ptr<int32_t>(); auto prob = a.ptr<float>(); auto count = a.ptr<int32_t>(); auto k = a.i32(), tail = a.i32();
        auto weight = a.ptr<float>(); auto stats = a.ptr<double>(); auto grad = a.ptr(); auto ldg = a.i64(); auto s = a.stream();
        return [=] { return picospec_distill_grad(z, dt, ld, rows, V, T, idx, prob, count, k, tail, weight, stats, grad, ldg, s); };
    });
}

// ---- the distillation loss on torch's tape, in native code: the engine runs the backward call in a thread of its own, which would have to wait for the
// interpreter twice (forward and backward of a small batch, on the host: 37 us with a Python function, of which torch takes 25 for any operator)

// A call that the library would refuse, or has refused.  Where no call of the binding answers it with its code - a backward call, in a thread of the engine's - it is an error like any other.
struct Refused : std::runtime_error {
    int code;
    explicit Refused(int code) : std::runtime_error("picospec error " + std::to_string(code) + ": " + picospec_strerror(code)), code(code) {}
};

int logits_code(const at::Tensor& t, int64_t& ld) {        // dtype code or error of rows2d
    if (t.dim() != 2 || !t.is_cuda()) throw Refused{PICOSPEC_EINVAL};
    if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) throw Refused{PICOSPEC_EDTYPE};
    if (t.size(0) != 0 && t.stride(1) != 1) throw Refused{PICOSPEC_EINVAL};
    ld = t.size(0) ? t.stride(0) : t.size(1);
    return t.scalar_type() == at::kFloat ? PICOSPEC_F32 : PICOSPEC_BF16;
}

bool dense(const at::Tensor& t, at::ScalarType type, const at::Tensor& z) { return t.scalar_type() == type && t.is_contiguous() && t.device() == z.device(); }

// the record's arrays are of the logits' rows and k entries each, without gaps
void check_record(const at::Tensor& z, const at::Tensor& idx, const at::Tensor& prob, const at::Tensor& count, int64_t k) {
    const int64_t rows = z.size(0);
    for (const at::Tensor* t : {&idx, &prob})
        if (t->dim() != 2 || t->size(0) != rows || t->size(1) != k) throw Refused{PICOSPEC_EINVAL};
    if (count.dim() != 1 || count.size(0) != rows) throw Refused{PICOSPEC_EINVAL};
    if (!dense(idx, at::kInt, z) || !dense(prob, at::kFloat, z) || !dense(count, at::kInt, z)) throw Refused{PICOSPEC_EINVAL};
}

struct DistillLoss : torch::autograd::Function<DistillLoss> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& z, const at::Tensor& idx, const at::Tensor& prob, const at::Tensor& count,
                                                  int64_t k, int64_t V, double T, int64_t tail) {
        int64_t ld;
        const int dt = logits_code(z, ld);
        const int64_t rows = z.size(0);
        check_record(z, idx, prob, count, k);
        if (V > z.size(1)) throw Refused{PICOSPEC_EINVAL};                                          // (a view's rows end before its stride does)
        const auto f32 = z.options().dtype(at::kFloat);
        at::Tensor loss = at::empty({rows}, f32), accept = at::empty({rows}, f32), stats = at::empty({rows, 4}, z.options().dtype(at::kDouble));
        const size_t bytes = picospec_scratch_bytes(PICOSPEC_CALL_DISTILL, dt, (int32_t)rows, 0, (int32_t)V, 0);
        const at::Tensor scratch = bytes ? at::empty({(int64_t)bytes}, z.options().dtype(at::kByte)) : at::Tensor();
        void* const stream = c10::hip::getCurrentHIPStream().stream();
        const int rc = in_library([&] { return picospec_distill(z.data_ptr(), dt, ld, (int32_t)rows, (int32_t)V, (float)T, idx.data_ptr<int32_t>(), prob.data_ptr<float>(), count.data_ptr<int32_t>(), (int32_t)k,
                                        (int)tail, nullptr, loss.data_ptr<float>(), accept.data_ptr<float>(), stats.data_ptr<double>(), nullptr, 0,
                                        bytes ? scratch.data_ptr() : nullptr, bytes, stream); });
        if (rc != PICOSPEC_OK) throw Refused{rc};
        ctx->save_for_backward({z, idx, prob, count, stats});
        ctx->saved_data["k"] = k;
        ctx->saved_data["V"] = V;
        ctx->saved_data["T"] = T;
        ctx->saved_data["tail"] = tail;
        ctx->mark_non_differentiable({accept});
        ctx->set_materialize_grads(false);
        return {loss, accept};
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        torch::autograd::variable_list out(8);
        if (!grads[0].defined()) return out;
        TORCH_CHECK(!at::GradMode::is_enabled(), "distill_loss is differentiable once");           // (create_graph: the kernel is not on the tape)
        const auto saved = ctx->get_saved_variables();
        const at::Tensor &z = saved[0], &idx = saved[1], &prob = saved[2], &count = saved[3], &stats = saved[4];
        const int64_t k = ctx->saved_data["k"].toInt(), V = ctx->saved_data["V"].toInt(), tail = ctx->saved_data["tail"].toInt();
        const double T = ctx->saved_data["T"].toDouble();
        int64_t ld;
        const int dt = logits_code(z, ld);
        const at::Tensor weight = grads[0].contiguous();                                            // (of a sum or mean over the rows: one value seen from every row)
        // (what a hook gives back for the saved tensors need not be what they were)
        check_record(z, idx, prob, count, k);
        if (V > z.size(1) || stats.dim() != 2 || stats.size(0) != z.size(0) || stats.size(1) != 4 || !dense(stats, at::kDouble, z)) throw Refused{PICOSPEC_EINVAL};
        if (weight.numel() != z.size(0) || !dense(weight, at::kFloat, z)) throw Refused{PICOSPEC_EINVAL};
        at::Tensor grad = at::empty(z.sizes(), z.options());
        if (z.size(1) > V) grad.slice(1, V).zero_();                                                // (columns behind the vocabulary are not read)
        void* const stream = c10::hip::getCurrentHIPStream().stream();
        const int rc = in_library([&] { return picospec_distill_grad(z.data_ptr(), dt, ld, (int32_t)z.size(0), (int32_t)V, (float)T, idx.data_ptr<int32_t>(), prob.data_ptr<float>(), count.data_ptr<int32_t>(), (int32_t)k,
                                             (int)tail, weight.data_ptr<float>(), stats.data_ptr<double>(), grad.data_ptr(), z.size(1), stream); });
        TORCH_CHECK(rc == PICOSPEC_OK, "picospec error ", rc, ": ", picospec_strerror(rc));
        out[0] = grad;
        return out;
    }
};

// distill_loss(logits, idx, prob, count, k, V, temperature, tail) -> (loss, accept), or an error code of the library
PyObject* n_distill_loss(PyObject*, PyObject* const* v, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        Args a{v, n};
        const at::Tensor* t[4];
        for (auto& x : t) x = &a.tensor();
        const int64_t k = a.i64(), V = a.i64();
        const double T = a.f32();
        const int64_t tail = a.i64();
        a.done();
        if (V < 1 || V > INT32_MAX || k < 1 || k > INT32_MAX || (tail != 0 && tail != 1)) throw Refused{PICOSPEC_EINVAL};
        auto out = DistillLoss::apply(*t[0], *t[1], *t[2], *t[3], k, V, T, tail);
        THPObjectPtr pair(PyTuple_New(2));
        if (!pair) return nullptr;
        for (int i = 0; i < 2; ++i) {
            PyObject* o = THPVariable_Wrap(out[i]);
            if (!o) return nullptr;
            PyTuple_SET_ITEM(pair.get(), i, o);
        }
        return pair.release();
    } catch (const Refused& r) {
        return PyLong_FromLong(r.code);
    } catch (const BadArgument& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// ---- adjusted logits, embeddings and clipped gradients.  These calls run on the current stream of their tensors' device, whichever device is current.

using c10::hip::getCurrentHIPStream;

at::Tensor optional_tensor(Args& a) {
    PyObject* o = a.next();
    if (o == Py_None) return at::Tensor();
    if (!THPVariable_Check(o)) throw BadArgument("a tensor or None is expected");
    return THPVariable_Unpack(o);
}

void refuse_unless(bool ok) { if (!ok) throw Refused{PICOSPEC_EINVAL}; }

// rows of V columns and more in the type of `z` and on its device; returns the stride of a row
int64_t rows_like(const at::Tensor& t, const at::Tensor& z, int64_t rows, int64_t V) {
    refuse_unless(t.dim() == 2 && t.size(0) == rows && t.size(1) >= V && t.device() == z.device());
    if (t.scalar_type() != z.scalar_type()) throw Refused{PICOSPEC_EDTYPE};
    int64_t ld;
    logits_code(t, ld);
    return rows <= 1 ? std::max(ld, V) : ld;
}

template <class T> const T* data(const at::Tensor& t) { return t.defined() ? static_cast<const T*>(t.data_ptr()) : nullptr; }

// a setting: a number for all sequences or a tensor with one for each
struct Setting { float all; at::Tensor each; };
Setting one_setting(Args& a) {
    PyObject* o = a.next();
    if (THPVariable_Check(o)) return {0.f, THPVariable_Unpack(o)};
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw BadArgument("");
    return {(float)v, at::Tensor()};
}

// What a call adjusts its rows by, checked against them
struct Adjustment {
    at::Tensor hist_tok, length, prompt, bias_off, bias_id, bias_value, mask, mask_row, seq_off, draft_tok;
    Setting repetition, presence, frequency;
    int64_t B = 0, ld_hist = 0, hist_cap = 0, n_draft = 0, n_bias = 0, n_masks = 0, ld_mask = 0;

    explicit Adjustment() = default;
    explicit Adjustment(Args& a) {
        hist_tok = optional_tensor(a); length = optional_tensor(a); prompt = optional_tensor(a);
        repetition = one_setting(a); presence = one_setting(a); frequency = one_setting(a);
        bias_off = optional_tensor(a); bias_id = optional_tensor(a); bias_value = optional_tensor(a);
        mask = optional_tensor(a); mask_row = optional_tensor(a); seq_off = optional_tensor(a); draft_tok = optional_tensor(a);
    }
    void check(const at::Tensor& z, int64_t V) {
        const int64_t rows = z.size(0);
        auto list = [&](const at::Tensor& t, at::ScalarType type, int64_t n) { refuse_unless(t.defined() && t.dim() == 1 && (n < 0 || t.numel() == n) && dense(t, type, z)); };
        refuse_unless(V >= 1 && V <= z.size(1) && rows <= INT32_MAX);
        if (V > INT32_MAX) throw Refused{PICOSPEC_EUNSUPPORTED};                                    // (the library's sizes have 32 bits)
        B = rows;
        if (seq_off.defined()) {
            list(seq_off, at::kInt, -1);
            list(draft_tok, at::kInt, -1);
            refuse_unless(seq_off.numel() >= 1 && draft_tok.numel() <= INT32_MAX);
            B = seq_off.numel() - 1;
            n_draft = draft_tok.numel();
        } else {
            refuse_unless(!draft_tok.defined());
        }
        if (hist_tok.defined()) {
            refuse_unless(hist_tok.dim() == 2 && hist_tok.size(0) == B && hist_tok.scalar_type() == at::kInt && hist_tok.device() == z.device());
            hist_cap = hist_tok.size(1);
            ld_hist = B > 1 ? hist_tok.stride(0) : hist_cap;
            refuse_unless(hist_cap <= INT32_MAX && (hist_cap <= 1 || hist_tok.stride(1) == 1));
            list(length, at::kInt, B);
            if (prompt.defined()) list(prompt, at::kInt, B);
        }
        for (const Setting* s : {&repetition, &presence, &frequency}) if (s->each.defined()) list(s->each, at::kFloat, B);
        if (bias_off.defined()) {
            list(bias_off, at::kInt, B + 1);
            list(bias_id, at::kInt, -1);
            list(bias_value, at::kFloat, bias_id.numel());
            refuse_unless(bias_id.numel() <= INT32_MAX);
            n_bias = bias_id.numel();
        }
        if (mask.defined()) {
            refuse_unless(mask.dim() == 2 && mask.scalar_type() == at::kInt && mask.device() == z.device() && mask.size(0) <= INT32_MAX && mask.size(1) >= (V + 31) / 32 && (mask.size(1) == 1 || mask.stride(1) == 1));
            n_masks = mask.size(0);
            ld_mask = n_masks > 1 ? mask.stride(0) : mask.size(1);
            if (mask_row.defined()) list(mask_row, at::kInt, rows);
            else refuse_unless(n_masks >= rows);
        } else {
            refuse_unless(!mask_row.defined());
        }
    }
    // whole: `out` is new, and rows that no sequence has are zeros in it
    int forward(const at::Tensor& z, int dt, int64_t ld, int64_t V, at::Tensor& out, int64_t ld_out, bool whole) const {
        void* const stream = getCurrentHIPStream().stream();
        return in_library([&] { return (whole ? picospec_adjust_whole : picospec_adjust)(z.data_ptr(), dt, ld, (int32_t)z.size(0), (int32_t)V, (int32_t)B, (int32_t)n_draft, data<int32_t>(seq_off), data<int32_t>(draft_tok),
                               data<int32_t>(hist_tok), ld_hist, (int32_t)hist_cap, data<int32_t>(length), data<int32_t>(prompt), repetition.all, presence.all, frequency.all,
                               data<float>(repetition.each), data<float>(presence.each), data<float>(frequency.each), data<int32_t>(bias_off), data<int32_t>(bias_id), data<float>(bias_value), (int32_t)n_bias,
                               data<uint32_t>(mask), ld_mask, (int32_t)n_masks, data<int32_t>(mask_row), out.data_ptr(), ld_out, stream); });
    }
    int backward(const at::Tensor& g, int64_t ld_g, const at::Tensor& z, int dt, int64_t ld, int64_t V, at::Tensor& out, int64_t ld_out, bool whole) const {
        void* const stream = getCurrentHIPStream().stream();
        return in_library([&] { return (whole ? picospec_adjust_grad_whole : picospec_adjust_grad)(g.data_ptr(), ld_g, z.data_ptr(), dt, ld, (int32_t)z.size(0), (int32_t)V, (int32_t)B, (int32_t)n_draft, data<int32_t>(seq_off), data<int32_t>(draft_tok),
                                    data<int32_t>(hist_tok), ld_hist, (int32_t)hist_cap, data<int32_t>(length), repetition.all, data<float>(repetition.each),
                                    data<uint32_t>(mask), ld_mask, (int32_t)n_masks, data<int32_t>(mask_row), out.data_ptr(), ld_out, stream); });
    }
};

// A tensor that a call is to write, or reads without a gradient for it, must not be part of what the tape records: a gradient that is taken later would leave the call out
void refuse_recorded(const at::Tensor& t) { refuse_unless(!(t.defined() && t.requires_grad() && at::GradMode::is_enabled())); }

// A tensor that a call has written in place: what the tape has saved of it is not what it was
void written(const at::Tensor& t) { if (!t.is_inference()) torch::autograd::impl::bump_version(t); }

// Runs `call(args)`, which returns a new reference; a refusal is returned as the library's error code
template <class F>
PyObject* answer(PyObject* const* v, Py_ssize_t n, F call) {
    HANDLE_TH_ERRORS
    try {
        Args a{v, n};
        return call(a);
    } catch (const Refused& r) {
        return PyLong_FromLong(r.code);
    } catch (const BadArgument& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

void check_code(int rc) { if (rc != PICOSPEC_OK) throw Refused{rc}; }

// adjust(logits, V, hist_tok, length, prompt, repetition, presence, frequency, bias_off, bias_id, bias_value, mask, mask_row, seq_off, draft_tok, grad, out) -> tensor or an error code; with a
// gradient its own
PyObject* n_adjust(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return answer(v, n, [](Args& a) {
        const at::Tensor z = a.tensor();
        const int64_t V = a.i64();
        Adjustment by(a);
        const at::Tensor grad = optional_tensor(a);
        at::Tensor out = optional_tensor(a);
        a.done();
        refuse_recorded(out);
        const bool given = out.defined();
        int64_t ld, ld_g = 0;
        const int dt = logits_code(z, ld);
        by.check(z, V);
        const int64_t rows = z.size(0);
        if (rows <= 1) ld = std::max(ld, V);
        if (grad.defined()) ld_g = rows_like(grad, z, rows, V);
        const c10::DeviceGuard guard(z.device());
        if (!given) out = at::empty({rows, V}, z.options());
        const int64_t ld_out = rows_like(out, z, rows, V);
        check_code(grad.defined() ? by.backward(grad, ld_g, z, dt, ld, V, out, ld_out, !given) : by.forward(z, dt, ld, V, out, ld_out, !given));
        if (given) written(out);
        return THPVariable_Wrap(out);
    });
}

struct AdjustFunction : torch::autograd::Function<AdjustFunction> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& z, Adjustment* by, int64_t V) {
        int64_t ld;
        const int dt = logits_code(z, ld);
        by->check(z, V);
        if (z.size(0) <= 1) ld = std::max(ld, V);
        const c10::DeviceGuard guard(z.device());
        at::Tensor out = at::empty({z.size(0), V}, z.options());
        check_code(by->forward(z, dt, ld, V, out, V, true));
        ctx->save_for_backward({z, by->hist_tok, by->length, by->repetition.each, by->mask, by->mask_row, by->seq_off, by->draft_tok});
        ctx->saved_data["V"] = V;
        ctx->saved_data["repetition"] = (double)by->repetition.all;
        return out;
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "adjust is differentiable once");                 // (create_graph: the kernel is not on the tape)
        const auto saved = ctx->get_saved_variables();
        const at::Tensor& z = saved[0];
        const int64_t V = ctx->saved_data["V"].toInt();
        Adjustment by;
        by.hist_tok = saved[1]; by.length = saved[2]; by.repetition = {(float)ctx->saved_data["repetition"].toDouble(), saved[3]};
        by.mask = saved[4]; by.mask_row = saved[5]; by.seq_off = saved[6]; by.draft_tok = saved[7];
        by.check(z, V);
        int64_t ld;
        const int dt = logits_code(z, ld);
        if (z.size(0) <= 1) ld = std::max(ld, V);
        const c10::DeviceGuard guard(z.device());
        at::Tensor out = at::empty(z.sizes(), z.options());
        if (z.size(1) > V) out.slice(1, V).zero_();                                                 // (columns behind the vocabulary are not read)
        const at::Tensor g = grads[0].contiguous();                                                 // (of a sum: one value seen from every place)
        rows_like(g, z, z.size(0), V);                                                              // (what a hook gives back for the logits need not have the rows that they had)
        check_code(by.backward(g, V, z, dt, ld, V, out, z.size(1), true));
        return {out, at::Tensor(), at::Tensor()};
    }
};

// adjust_on_tape(logits, V, ... as adjust, draft_tok) -> tensor or an error code
PyObject* n_adjust_on_tape(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return answer(v, n, [](Args& a) {
        const at::Tensor z = a.tensor();
        const int64_t V = a.i64();
        Adjustment by(a);
        a.done();
        for (const at::Tensor* t : {&by.repetition.each, &by.presence.each, &by.frequency.each, &by.bias_value}) refuse_recorded(*t);      // (they would have no gradient)
        return THPVariable_Wrap(AdjustFunction::apply(z, &by, V));
    });
}

struct Table { int dt; int64_t ld, V, d; };
Table check_table(const at::Tensor& t) {
    int64_t ld;
    const int dt = logits_code(t, ld);
    refuse_unless(t.size(0) >= 1 && t.size(0) <= INT32_MAX && t.size(1) >= 1 && t.size(1) <= INT32_MAX);
    return {dt, t.size(0) == 1 ? std::max(ld, t.size(1)) : ld, t.size(0), t.size(1)};
}

at::Tensor embed(const at::Tensor& table, const at::Tensor& tok, float scale, at::Tensor out) {
    const Table t = check_table(table);
    refuse_unless(dense(tok, at::kInt, table) && tok.numel() <= INT32_MAX);
    const int64_t n = tok.numel();
    const c10::DeviceGuard guard(table.device());
    int64_t ld_out = t.d;
    if (out.defined()) {
        refuse_unless(out.dim() == 2 && out.size(1) == t.d);
        ld_out = rows_like(out, table, n, t.d);
    } else {
        auto sizes = tok.sizes().vec();
        sizes.push_back(t.d);
        out = at::empty(sizes, table.options());
    }
    void* const stream = getCurrentHIPStream().stream();
    check_code(in_library([&] { return picospec_embed(table.data_ptr(), t.dt, t.ld, (int32_t)t.V, (int32_t)t.d, data<int32_t>(tok), (int32_t)n, scale, out.data_ptr(), ld_out, stream); }));
    return out;
}

at::Tensor embed_grad(at::Tensor g, const at::Tensor& tok, int64_t V, float scale, int accumulate, at::Tensor out) {
    refuse_unless(g.is_cuda() && g.dim() == tok.dim() + 1 && g.sizes().slice(0, tok.dim()) == tok.sizes() && V >= 1 && V <= INT32_MAX);
    const int64_t n = tok.numel(), d = g.size(-1);
    refuse_unless(n <= INT32_MAX && d >= 1 && d <= INT32_MAX);
    const c10::DeviceGuard guard(g.device());
    if (g.dim() != 2) g = g.reshape({n, d});
    refuse_unless(dense(tok, at::kInt, g));
    int64_t ld;
    const int dt = logits_code(g, ld);
    if (n <= 1) ld = std::max(ld, d);
    refuse_unless(out.defined() || !accumulate);
    if (!out.defined()) out = at::empty({V, d}, g.options());
    refuse_unless(out.dim() == 2 && out.size(0) == V && out.size(1) == d && out.device() == g.device());
    const Table t = check_table(out);
    const size_t bytes = picospec_workspace_bytes(PICOSPEC_CALL_EMBED_GRAD, dt, (int32_t)n, (int32_t)V, (int32_t)d);
    const at::Tensor scratch = at::empty({(int64_t)std::max<size_t>(bytes, 16)}, g.options().dtype(at::kByte));
    void* const stream = getCurrentHIPStream().stream();
    check_code(in_library([&] { return picospec_embed_grad(g.data_ptr(), dt, ld, (int32_t)n, data<int32_t>(tok), (int32_t)V, (int32_t)d, scale, accumulate, out.data_ptr(), t.dt, t.ld,
                                   scratch.data_ptr(), (size_t)scratch.nbytes(), stream); }));
    return out;
}

// embed(table, tok, scale, out) -> rows or an error code
PyObject* n_embed(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return answer(v, n, [](Args& a) {
        const at::Tensor table = a.tensor(), tok = a.tensor();
        const float scale = a.f32();
        const at::Tensor out = optional_tensor(a);
        a.done();
        refuse_recorded(out);
        const at::Tensor rows = embed(table, tok, scale, out);
        if (out.defined()) written(out);
        return THPVariable_Wrap(rows);
    });
}

// embed_grad(grad, tok, V, scale, accumulate, out) -> the table's gradient or an error code
PyObject* n_embed_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return answer(v, n, [](Args& a) {
        const at::Tensor g = a.tensor(), tok = a.tensor();
        const int64_t V = a.i64();
        const float scale = a.f32();
        const int accumulate = a.i32();
        const at::Tensor out = optional_tensor(a);
        a.done();
        refuse_recorded(out);
        const at::Tensor sums = embed_grad(g, tok, V, scale, accumulate, out);
        if (out.defined()) written(out);
        return THPVariable_Wrap(sums);
    });
}

struct EmbedFunction : torch::autograd::Function<EmbedFunction> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& table, const at::Tensor& tok, double scale) {
        ctx->save_for_backward({tok});
        ctx->saved_data["V"] = table.size(0);
        ctx->saved_data["scale"] = scale;
        return embed(table, tok, (float)scale, at::Tensor());
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "embed is differentiable once");                   // (create_graph: the kernel is not on the tape)
        const auto saved = ctx->get_saved_variables();
        return {embed_grad(grads[0].contiguous(), saved[0], ctx->saved_data["V"].toInt(), (float)ctx->saved_data["scale"].toDouble(), 0, at::Tensor()), at::Tensor(), at::Tensor()};
    }
};

// embed_on_tape(table, tok, scale) -> rows or an error code
PyObject* n_embed_on_tape(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return answer(v, n, [](Args& a) {
        const at::Tensor table = a.tensor(), tok = a.tensor();
        const double scale = a.f32();
        a.done();
        if (table.dim() != 2) throw Refused{PICOSPEC_EINVAL};
        return THPVariable_Wrap(EmbedFunction::apply(table, tok, scale));
    });
}

// clip_grad(grads, max_norm, out) -> norm [1] or an error code; lists or tuples of tensors, out None: in place
PyObject* n_clip_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return answer(v, n, [](Args& a) {
        PyObject* const given = a.next();
        const float max_norm = a.f32();
        PyObject* const given_outs = a.next();
        a.done();
        // (as tuples: a list may be another one after the call, which gives the interpreter's lock up)
        auto sequence = [](PyObject* o) {
            if (!PyList_Check(o) && !PyTuple_Check(o)) throw BadArgument("a list or tuple of tensors is expected");
            PyObject* const t = PySequence_Tuple(o);
            if (!t) throw BadArgument("");
            return t;
        };
        const THPObjectPtr grads(sequence(given)), outputs(given_outs == Py_None ? nullptr : sequence(given_outs));
        const bool apart = outputs.get() != nullptr;
        const Py_ssize_t count = PyTuple_GET_SIZE(grads.get());
        refuse_unless(count <= INT32_MAX && (!apart || PyTuple_GET_SIZE(outputs.get()) == count));
        auto at_place = [](const THPObjectPtr& o, Py_ssize_t i) -> const at::Tensor& {
            PyObject* t = PyTuple_GET_ITEM(o.get(), i);
            if (!THPVariable_Check(t)) throw BadArgument("a list or tuple of tensors is expected");
            return THPVariable_Unpack(t);
        };
        c10::SmallVector<const void*, 128> g;
        c10::SmallVector<void*, 128> o;
        c10::SmallVector<int64_t, 128> numel;
        c10::SmallVector<int32_t, 128> dtypes;
        at::Tensor like;
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor& t = at_place(grads, i);
            refuse_unless(t.layout() == at::kStrided && t.is_cuda() && (!like.defined() || t.device() == like.device()));
            if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) throw Refused{PICOSPEC_EDTYPE};
            refuse_unless(t.is_non_overlapping_and_dense());
            if (!like.defined()) like = t;
            g.push_back(t.data_ptr());
            numel.push_back(t.numel());
            dtypes.push_back(t.scalar_type() == at::kFloat ? PICOSPEC_F32 : PICOSPEC_BF16);
            if (!apart) continue;
            const at::Tensor& to = at_place(outputs, i);
            refuse_recorded(to);
            refuse_unless(to.layout() == at::kStrided && to.device() == t.device() && to.sizes() == t.sizes() && to.strides() == t.strides());
            if (to.scalar_type() != t.scalar_type()) throw Refused{PICOSPEC_EDTYPE};
            o.push_back(to.data_ptr());
        }
        const c10::OptionalDeviceGuard guard(like.defined() ? c10::optional<at::Device>(like.device()) : c10::nullopt);
        const auto f32 = at::TensorOptions().dtype(at::kFloat).device(like.defined() ? like.device() : at::Device(at::kCUDA));
        at::Tensor norm = at::empty({1}, f32);
        const size_t bytes = picospec_workspace_bytes(PICOSPEC_CALL_CLIP_GRAD, 0, (int32_t)count, 1, 0);
        const at::Tensor scratch = at::empty({(int64_t)std::max<size_t>(bytes, 16)}, f32.dtype(at::kByte));
        void* const stream = getCurrentHIPStream().stream();
        check_code(in_library([&] { return picospec_clip_grad((int32_t)count, g.data(), apart ? o.data() : nullptr, numel.data(), dtypes.data(), max_norm, norm.data_ptr<float>(),
                                      scratch.data_ptr(), (size_t)scratch.nbytes(), stream); }));
        for (Py_ssize_t i = 0; i < count && (apart || !std::isinf(max_norm)); ++i) written(at_place(apart ? outputs : grads, i));
        return THPVariable_Wrap(norm);
    });
}

// rows2d(tensor) -> (dtype code, stride of a row, rows), or an error code of the library: a 2-d device tensor whose rows are
// contiguous (the strides of a tensor without rows mean nothing)
PyObject* n_rows2d(PyObject*, PyObject* o) {
    HANDLE_TH_ERRORS
    if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "a tensor is expected"); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.dim() != 2 || !t.is_cuda()) return PyLong_FromLong(PICOSPEC_EINVAL);
    int dt;
    if (t.scalar_type() == at::kFloat) dt = PICOSPEC_F32;
    else if (t.scalar_type() == at::kBFloat16) dt = PICOSPEC_BF16;
    else return PyLong_FromLong(t.size(0) != 0 && t.stride(1) != 1 ? PICOSPEC_EINVAL : PICOSPEC_EDTYPE);
    const int64_t rows = t.size(0);
    if (rows != 0 && t.stride(1) != 1) return PyLong_FromLong(PICOSPEC_EINVAL);
    return Py_BuildValue("(iLL)", dt, (long long)(rows ? t.stride(0) : t.size(1)), (long long)rows);
    END_HANDLE_TH_ERRORS
}

// distill_inputs(logits, idx, prob, count, k, weight or None) -> rows2d(logits), or an error code where record or weights are not the rows'
PyObject* n_distill_inputs(PyObject*, PyObject* const* v, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        Args a{v, n};
        const at::Tensor &z = a.tensor(), &idx = a.tensor(), &prob = a.tensor(), &count = a.tensor();
        const int64_t k = a.i64();
        PyObject* const w = a.next();
        a.done();
        int64_t ld;
        const int dt = logits_code(z, ld);
        check_record(z, idx, prob, count, k);
        if (w != Py_None) {
            if (!THPVariable_Check(w)) throw BadArgument("a tensor or None is expected");
            const at::Tensor& t = THPVariable_Unpack(w);
            if (t.numel() != z.size(0) || !dense(t, at::kFloat, z)) throw Refused{PICOSPEC_EINVAL};
        }
        return Py_BuildValue("(iLL)", dt, (long long)ld, (long long)z.size(0));
    } catch (const Refused& r) {
        return PyLong_FromLong(r.code);
    } catch (const BadArgument& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

at::TensorOptions like(PyObject* o, at::ScalarType type) { return at::TensorOptions().dtype(type).device(THPVariable_Unpack(o).device()); }

// scratch_bytes(which, dtype, n_draft, B, V, k) -> picospec_scratch_bytes(...)
PyObject* n_scratch_bytes(PyObject*, PyObject* const* v, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        Args a{v, n};
        const int which = a.i32(), dt = a.i32(), N = a.i32(), B = a.i32(), V = a.i32(), k = a.i32();
        a.done();
        return PyLong_FromSize_t(picospec_scratch_bytes(which, dt, N, B, V, k));
    } catch (const BadArgument& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// scratch(like, which, dtype, n_draft, B, V, k[, given]) -> uint8 tensor of picospec_one_launch_bytes(...) bytes.  None where that is
// 0, where the caller's workspace `given` holds as many, and where the library refuses that one (it still does).
PyObject* n_scratch(PyObject*, PyObject* const* v, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        if ((n != 7 && n != 8) || !THPVariable_Check(v[0])) throw BadArgument("scratch(tensor, which, dtype, n_draft, B, V, k[, given])");
        Args a{v, n, 1};
        const int which = a.i32(), dt = a.i32(), N = a.i32(), B = a.i32(), V = a.i32(), k = a.i32();
        const size_t bytes = picospec_scratch_bytes(which, dt, N, B, V, k);
        if (!bytes) Py_RETURN_NONE;
        if (n == 8) {
            const Args::Buffer given = a.buffer();
            if (given.p && (given.bytes >= bytes || ((uintptr_t)given.p & 15u) || given.bytes < picospec_workspace_bytes(which, dt, N + B, V, 0))) Py_RETURN_NONE;
        }
        return THPVariable_Wrap(at::empty({(int64_t)picospec_one_launch_bytes(which, dt, N, B, V, k)}, like(v[0], at::kByte)));
    } catch (const BadArgument& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// empty(like, codes, size, ...) -> one tensor per letter of `codes` (i int32, l int64, f float32, d float64, b uint8) on the device of
// `like`; a size is an int (1-d) or a tuple of two.  Outputs of up to kShared bytes share one allocation, each from a 512-byte boundary of it
// on, as slices of a tensor do: an allocation costs 0.45 to 0.85 us, a slice 0.15 (the eight outputs of an unpacked downlink message of 32
// records of 256: 2.1 us, each from torch.empty 6.8).  All of it lives as long as any of them, so larger ones, next to which an allocation is cheap to make and
// dear to keep, have their own.
PyObject* n_empty(PyObject*, PyObject* const* v, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    constexpr Py_ssize_t kMost = 16;
    constexpr int64_t kShared = 64 * 1024;
    Py_ssize_t len = 0;
    const char* codes = n >= 2 && THPVariable_Check(v[0]) ? PyUnicode_AsUTF8AndSize(v[1], &len) : nullptr;
    if (!codes || n != len + 2 || len > kMost) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "empty(tensor, codes, size, ...)"); return nullptr; }
    int64_t dims[kMost][2], bytes[kMost], shared = 0;
    int nd[kMost];
    for (Py_ssize_t i = 0; i < len; ++i) {
        PyObject* s = v[2 + i];
        nd[i] = PyTuple_Check(s) && PyTuple_GET_SIZE(s) == 2 ? 2 : 1;
        dims[i][0] = PyLong_AsLongLong(nd[i] == 2 ? PyTuple_GET_ITEM(s, 0) : s);
        dims[i][1] = nd[i] == 2 ? PyLong_AsLongLong(PyTuple_GET_ITEM(s, 1)) : 1;
        if (PyErr_Occurred()) return nullptr;
        if (dims[i][0] < 0 || dims[i][1] < 0 || __builtin_mul_overflow(dims[i][0], dims[i][1], &bytes[i]) || bytes[i] > (int64_t(1) << 56)) { PyErr_SetString(PyExc_RuntimeError, "empty: a size is out of range"); return nullptr; }
        bytes[i] *= codes[i] == 'l' || codes[i] == 'd' ? 8 : codes[i] == 'b' ? 1 : 4;
        if (bytes[i] <= kShared) shared += (bytes[i] + 511) / 512 * 512;
    }
    THPObjectPtr out(PyTuple_New(len));
    if (!out) return nullptr;
    at::Tensor block;
    int64_t at_byte = 0;
    for (Py_ssize_t i = 0; i < len; ++i) {
        const at::ScalarType type = codes[i] == 'i' ? at::kInt : codes[i] == 'l' ? at::kLong : codes[i] == 'b' ? at::kByte : codes[i] == 'd' ? at::kDouble : at::kFloat;
        at::Tensor piece;
        if (bytes[i] > kShared) {
            piece = at::empty(at::IntArrayRef(dims[i], nd[i]), like(v[0], type));
        } else {
            if (!block.defined()) block = at::empty({shared}, like(v[0], at::kByte));
            piece = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(block.storage()), block.key_set(), c10::scalarTypeToTypeMeta(type));
            piece.unsafeGetTensorImpl()->set_storage_offset(at_byte / (int64_t)c10::elementSize(type));
            piece.unsafeGetTensorImpl()->set_sizes_contiguous(at::IntArrayRef(dims[i], nd[i]));
            at_byte += (bytes[i] + 511) / 512 * 512;
        }
        PyObject* t = THPVariable_Wrap(piece);
        if (!t) return nullptr;
        PyTuple_SET_ITEM(out.get(), i, t);
    }
    return out.release();
    END_HANDLE_TH_ERRORS
}

#define FAST(name, f) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    FAST("compress", n_compress), FAST("sample_draft", n_sample_draft), FAST("verify", n_verify), FAST("verify_range", n_verify_range),
    FAST("round", n_round), FAST("verify_sample", n_verify_sample), FAST("verify_sample_static", n_verify_sample_static),
    FAST("sample_residual", n_sample_residual<picospec_sample_residual>), FAST("sample_residual_ws", n_sample_residual<picospec_sample_residual_ws>), FAST("row_stats", n_row_stats), FAST("compress_rejected", n_compress_rejected),
    FAST("resample_sparse", n_resample_sparse), FAST("pack_downlink", n_pack_downlink), FAST("unpack_downlink", n_unpack_downlink),
    FAST("pack_uplink", n_pack_uplink), FAST("unpack_uplink", n_unpack_uplink), FAST("sample", n_sample), FAST("distill", n_distill), FAST("distill_grad", n_distill_grad), FAST("distill_loss", n_distill_loss), FAST("distill_inputs", n_distill_inputs), FAST("adjust", n_adjust), FAST("adjust_on_tape", n_adjust_on_tape), FAST("embed", n_embed), FAST("embed_grad", n_embed_grad),
    FAST("embed_on_tape", n_embed_on_tape), FAST("clip_grad", n_clip_grad), FAST("scratch_bytes", n_scratch_bytes), FAST("scratch", n_scratch), FAST("empty", n_empty),
    {"rows2d", (PyCFunction)n_rows2d, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
