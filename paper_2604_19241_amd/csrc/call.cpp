// The host side of the calls that are shorter on the GPU than in Python: checks of the tensors, allocation of the outputs and the call itself.
// A pass of a few tokens is two launches of 5 us; the same in Python (binding.py marshals every other entry point) took 12.6 us for a
// projection and 21 for a router's loss with its gradient, most of it property by property; here 8.4 and 13.1 (one token; 256 tokens of 8 experts).
// Knows no HIP: streams and the library's functions come as addresses from binding.py.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/uniep_moe.h"

namespace {

decltype(&moe_adapter_plan) p_adapter_plan;
decltype(&moe_adapter_forward) p_adapter_forward;
decltype(&moe_adapter_backward) p_adapter_backward;
decltype(&moe_balance_forward) p_balance_forward;
decltype(&moe_balance_backward) p_balance_backward;
decltype(&moe_adapter_workspace_bytes) p_adapter_bytes;
decltype(&moe_balance_workspace_bytes) p_balance_bytes;

struct Refused {};   // a Python exception is set

[[noreturn]] void refuse(const char* name, const char* what) {
    PyErr_Format(PyExc_AssertionError, "%s: %s", name, what);
    throw Refused{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(name, "expected a tensor");
    return THPVariable_Unpack(o);
}
at::Tensor made(const at::Tensor& like, at::ScalarType type, at::IntArrayRef sizes) { return at::empty(sizes, like.options().dtype(type)); }

// Tensor arguments: on the GPU that the call's first one is on (a kernel that is launched there would read another's memory over the links, or not at all), of the type and the
// sizes that are asked for.
struct On {
    const at::Tensor& first;
    On(PyObject* o, const char* name) : first(tensor(o, name)) { here(first, name); }
    void here(const at::Tensor& t, const char* name) const {
        if (!t.is_cuda()) refuse(name, "expected a tensor on the GPU");
        if (t.get_device() != first.get_device()) refuse(name, "on another GPU than the call's other tensors");
    }
    void check(const at::Tensor& t, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes) const {
        here(t, name);
        if (t.scalar_type() != type) refuse(name, "type");
        if (t.sizes() != at::IntArrayRef(sizes.begin(), sizes.size())) refuse(name, "sizes");
    }
    void* dense(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes) const {
        const at::Tensor& t = tensor(o, name);
        check(t, name, type, sizes);
        if (!t.is_contiguous()) refuse(name, "expected a contiguous tensor");
        return t.data_ptr();
    }
    void* optional(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes) const {
        return o == Py_None ? nullptr : dense(o, name, type, sizes);
    }
    // Rows of `width` that may be parts of wider ones; ld = elements from one to the next.
    void* rows(PyObject* o, const char* name, int64_t n, int64_t width, int64_t* ld) const {
        const at::Tensor& t = tensor(o, name);
        check(t, name, at::kBFloat16, {n, width});
        if (t.stride(1) != 1 && width > 1) refuse(name, "expected rows without gaps");
        *ld = n > 1 ? t.stride(0) : width;
        return t.data_ptr();
    }
    // The caller's output, or a new one.
    at::Tensor output(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes) const {
        if (o == Py_None) return made(first, type, at::IntArrayRef(sizes.begin(), sizes.size()));
        dense(o, name, type, sizes);
        return THPVariable_Unpack(o);
    }
};
struct Workspace {
    at::Tensor own;
    void* p;
    size_t bytes;
    Workspace(PyObject* o, const On& on, size_t need) {
        if (o == Py_None) own = made(on.first, at::kByte, {(int64_t)(need < 256 ? 256 : need)});
        const at::Tensor& t = o == Py_None ? own : tensor(o, "ws");
        on.here(t, "ws");
        if (t.scalar_type() != at::kByte || !t.is_contiguous()) refuse("ws", "expected contiguous bytes");
        p = t.data_ptr();
        bytes = (size_t)t.numel();
    }
};
void* stream_of(PyObject* o) {
    void* p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) throw Refused{};
    return p;
}
template <class S>
S shape_at(PyObject* o) {   // address of the ctypes structure
    const void* p = PyLong_AsVoidPtr(o);
    if (!p) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no shape");
        throw Refused{};
    }
    return *(const S*)p;
}
// The results, or the library's code as an int.
PyObject* code_of(int rc) { return PyLong_FromLong(rc); }
PyObject* wrapped(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* wrapped(std::initializer_list<at::Tensor> ts) {
    PyObject* out = PyTuple_New((Py_ssize_t)ts.size());
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) PyTuple_SET_ITEM(out, i++, THPVariable_Wrap(t));
    return out;
}
// A call of the library: other threads of the program run meanwhile, as behind ctypes.
template <class F>
int call(F f) {
    PyThreadState* const state = PyEval_SaveThread();
    const int rc = f();
    PyEval_RestoreThread(state);
    return rc;
}
template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments", want);
        return nullptr;
    }
    try {
        return f();
    } catch (const Refused&) {
        return nullptr;
    } catch (...) {   // as torch's own functions raise it: torch.OutOfMemoryError for an allocation that failed
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

// shape, ids, stream -> table or None
PyObject* adapter_plan(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 3, [&]() -> PyObject* {
        const auto s = shape_at<moe_adapter_shape_t>(v[0]);
        const On on(v[1], "ids");
        const void* ids = on.dense(v[1], "ids", at::kInt, {s.T});
        size_t need = 0;
        int rc = p_adapter_bytes(&s, nullptr, &need);
        if (rc != MOE_OK) return code_of(rc);
        if (need == 0) Py_RETURN_NONE;
        const at::Tensor table = made(on.first, at::kInt, {(int64_t)(need / 4)});
        void* const stream = stream_of(v[2]);
        rc = call([&] { return p_adapter_plan(&s, (const int32_t*)ids, table.data_ptr(), need, stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped(table);
    });
}

struct Operands {
    const void *w, *a, *b, *ids, *table;
    const float* scale;
    // w, a, b, scale, ids, table, adapters of the table
    Operands(const On& on, const moe_adapter_shape_t& s, PyObject* const* v) {
        w = on.dense(v[0], "w", at::kBFloat16, {s.K, s.N});
        a = on.dense(v[1], "a", at::kBFloat16, {s.adapters, s.rank, s.K});
        b = on.dense(v[2], "b", at::kBFloat16, {s.adapters, s.rank, s.N});
        scale = (const float*)on.optional(v[3], "scale", at::kFloat, {s.adapters});
        ids = on.dense(v[4], "ids", at::kInt, {s.T});
        table = nullptr;
        if (v[5] != Py_None) {
            const at::Tensor& t = tensor(v[5], "plan");
            if (PyLong_AsLong(v[6]) != s.adapters) refuse("plan", "made for another number of adapters");
            // (the kernels take token numbers from it: one of another batch would have them read elsewhere)
            on.here(t, "plan");
            if (t.scalar_type() != at::kInt || !t.is_contiguous()) refuse("plan", "expected a contiguous table of int32");
            moe_adapter_shape_t widest = s;   // up to 512 tokens some widths read no plan, and a plan serves them all
            if (s.T <= 512) widest.K = widest.N = 1 << 16;
            size_t need = 0;
            if (p_adapter_bytes(&widest, nullptr, &need) == MOE_OK && t.numel() != (int64_t)(need / 4))   // (else the call refuses the shape)
                refuse("plan", "made for another number of tokens");
            table = t.data_ptr();
        }
    }
};

// shape, x, w, a, b, scale, ids, table, adapters, fp32, h, y, ws, stream -> y
PyObject* adapter_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 14, [&]() -> PyObject* {
        const auto s = shape_at<moe_adapter_shape_t>(v[0]);
        const On on(v[1], "x");
        int64_t ldx;
        const void* x = on.rows(v[1], "x", s.T, s.K, &ldx);
        const Operands o(on, s, v + 2);
        const bool f32 = v[9] == Py_True;
        void* h = on.optional(v[10], "h", at::kFloat, {s.T, s.rank});
        const at::Tensor y = on.output(v[11], "y", f32 ? at::kFloat : at::kBFloat16, {s.T, s.N});
        size_t need = 0;
        int rc = v[12] == Py_None ? p_adapter_bytes(&s, &need, nullptr) : MOE_OK;
        if (rc != MOE_OK) return code_of(rc);
        const Workspace ws(v[12], on, need);
        void* const stream = stream_of(v[13]);
        rc = call([&] {
            return p_adapter_forward(&s, x, ldx, o.w, o.a, o.b, o.scale, (const int32_t*)o.ids, o.table, y.data_ptr(), f32, (float*)h, ws.p, ws.bytes, stream);
        });
        return rc != MOE_OK ? code_of(rc) : wrapped(y);
    });
}

// shape, dy, x, w, a, b, scale, ids, table, adapters, h, dx, da, db, ws, stream -> (dx, da, db)
PyObject* adapter_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 16, [&]() -> PyObject* {
        const auto s = shape_at<moe_adapter_shape_t>(v[0]);
        const On on(v[2], "x");
        int64_t lddy, ldx;
        const void* dy = on.rows(v[1], "dy", s.T, s.N, &lddy);
        const void* x = on.rows(v[2], "x", s.T, s.K, &ldx);
        const Operands o(on, s, v + 3);
        const void* h = on.dense(v[10], "h", at::kFloat, {s.T, s.rank});
        const at::Tensor dx = on.output(v[11], "dx", at::kBFloat16, {s.T, s.K});
        const at::Tensor da = on.output(v[12], "da", at::kFloat, {s.adapters, s.rank, s.K});
        const at::Tensor db = on.output(v[13], "db", at::kFloat, {s.adapters, s.rank, s.N});
        size_t need = 0;
        int rc = v[14] == Py_None ? p_adapter_bytes(&s, &need, nullptr) : MOE_OK;
        if (rc != MOE_OK) return code_of(rc);
        const Workspace ws(v[14], on, need);
        void* const stream = stream_of(v[15]);
        rc = call([&] {
            return p_adapter_backward(&s, dy, lddy, x, ldx, o.w, o.a, o.b, o.scale, (const int32_t*)o.ids, o.table, (const float*)h, dx.data_ptr(),
                                      (float*)da.data_ptr(), (float*)db.data_ptr(), ws.p, ws.bytes, stream);
        });
        return rc != MOE_OK ? code_of(rc) : wrapped({dx, da, db});
    });
}

struct BalanceInputs {
    const float* logits;
    const int32_t *idx, *offsets;
    // logits, topk_idx, seq_offsets
    BalanceInputs(const On& on, const moe_balance_shape_t& s, PyObject* const* v) {
        logits = (const float*)on.dense(v[0], "logits", at::kFloat, {s.T, s.E});
        idx = (const int32_t*)on.dense(v[1], "topk_idx", at::kInt, {s.T, s.k});
        offsets = (const int32_t*)on.optional(v[2], "seq_offsets", at::kInt, {s.seqs + 1});
    }
};

// shape, logits, topk_idx, seq_offsets, mask, ws, stream -> (loss, counts, tokens, prob_sums, lse)
PyObject* balance_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject* {
        const auto s = shape_at<moe_balance_shape_t>(v[0]);
        const On on(v[1], "logits");
        const BalanceInputs in(on, s, v + 1);
        const at::Tensor& like = on.first;
        const uint8_t* mask = nullptr;
        if (v[4] != Py_None)
            mask = (const uint8_t*)on.dense(v[4], "mask", tensor(v[4], "mask").scalar_type() == at::kByte ? at::kByte : at::kBool, {s.T});
        const at::Tensor loss = made(like, at::kFloat, {3}), counts = made(like, at::kInt, {s.seqs, s.E}), tokens = made(like, at::kInt, {s.seqs + 1}),
                         sums = made(like, at::kFloat, {s.seqs, s.E}), lse = made(like, at::kFloat, {s.T});
        size_t need = 0;
        int rc = v[5] == Py_None ? p_balance_bytes(&s, &need) : MOE_OK;
        if (rc != MOE_OK) return code_of(rc);
        const Workspace ws(v[5], on, need);
        const moe_balance_stats_t out = {(float*)loss.data_ptr(), (int32_t*)counts.data_ptr(), (int32_t*)tokens.data_ptr(), (float*)sums.data_ptr(),
                                         (float*)lse.data_ptr()};
        void* const stream = stream_of(v[6]);
        rc = call([&] { return p_balance_forward(&s, in.logits, in.idx, in.offsets, mask, &out, ws.p, ws.bytes, stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped({loss, counts, tokens, sums, lse});
    });
}

// shape, logits, topk_idx, seq_offsets, counts, tokens, lse, topk_w, dtopk_w, dloss, bf16, out, stream -> dlogits
PyObject* balance_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> PyObject* {
        const auto s = shape_at<moe_balance_shape_t>(v[0]);
        const On on(v[1], "logits");
        const BalanceInputs in(on, s, v + 1);
        const moe_balance_stats_t st = {nullptr, (int32_t*)on.dense(v[4], "stats.counts", at::kInt, {s.seqs, s.E}),
                                        (int32_t*)on.dense(v[5], "stats.tokens", at::kInt, {s.seqs + 1}), nullptr,
                                        (float*)on.dense(v[6], "stats.lse", at::kFloat, {s.T})};
        const float* w = (const float*)on.optional(v[7], "topk_w", at::kFloat, {s.T, s.k});
        const float* dw = (const float*)on.optional(v[8], "dtopk_w", at::kFloat, {s.T, s.k});
        const at::Tensor& u = tensor(v[9], "dloss");
        on.here(u, "dloss");
        if (u.scalar_type() != at::kFloat || u.numel() != 1) refuse("dloss", "expected one fp32 value");
        const bool bf16 = v[10] == Py_True;
        const at::Tensor d = on.output(v[11], "out", bf16 ? at::kBFloat16 : at::kFloat, {s.T, s.E});
        void* const stream = stream_of(v[12]);
        const int rc = call([&] { return p_balance_backward(&s, in.logits, in.idx, in.offsets, &st, w, dw, (const float*)u.data_ptr(), d.data_ptr(), bf16, stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped(d);
    });
}

// addresses of the library's functions, in the order of the pointers above
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject* {
        void* f[7];
        for (int i = 0; i < 7; ++i) f[i] = stream_of(v[i]);
        p_adapter_plan = (decltype(p_adapter_plan))f[0];
        p_adapter_forward = (decltype(p_adapter_forward))f[1];
        p_adapter_backward = (decltype(p_adapter_backward))f[2];
        p_balance_forward = (decltype(p_balance_forward))f[3];
        p_balance_backward = (decltype(p_balance_backward))f[4];
        p_adapter_bytes = (decltype(p_adapter_bytes))f[5];
        p_balance_bytes = (decltype(p_balance_bytes))f[6];
        Py_RETURN_NONE;
    });
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(adapter_plan), FAST(adapter_forward), FAST(adapter_backward), FAST(balance_forward), FAST(balance_backward), FAST(bind),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() { return PyModule_Create(&module); }
