// The host side of the calls that are shorter on the GPU than in Python: checks of the tensors, allocation of the outputs and the call itself.
// A pass of a few tokens is two launches of 5 us; the same in Python (binding.py marshals every other entry point) took 12.6 us for a
// projection and 21 for a router's loss with its gradient, most of it property by property; here 8.4 and 13.1 (one token; 256 tokens of 8 experts).
// Knows no HIP: streams and the library's functions come as addresses from binding.py.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "../../include/uniep_moe.h"

namespace {

decltype(&moe_adapter_plan) p_adapter_plan;
decltype(&moe_adapter_forward) p_adapter_forward;
decltype(&moe_adapter_backward) p_adapter_backward;
decltype(&moe_balance_forward) p_balance_forward;
decltype(&moe_balance_backward) p_balance_backward;
decltype(&moe_adapter_workspace_bytes) p_adapter_bytes;
decltype(&moe_balance_workspace_bytes) p_balance_bytes;
decltype(&moe_dispatch_forward) p_dispatch_forward;
decltype(&moe_dispatch_backward) p_dispatch_backward;
decltype(&moe_combine_forward) p_combine_forward;
decltype(&moe_combine_backward) p_combine_backward;
decltype(&moe_saved_layout) p_saved_layout;
decltype(&moe_saved_pack) p_saved_pack;
decltype(&moe_saved_unpack) p_saved_unpack;
decltype(&moe_mx_quantize) p_mx_quantize;
decltype(&moe_mx_quantize_weights) p_mx_quantize_weights;
decltype(&moe_mx_values) p_mx_values;
decltype(&moe_mx_product) p_mx_product;
decltype(&moe_mx_gate_up) p_mx_gate_up;

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
    c10::OptionalDeviceGuard current;   // its GPU is the current one during the call, where there are several
    On(PyObject* o, const char* name) : first(tensor(o, name)) {
        here(first, name);
        static const bool several = c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->deviceCount() > 1;
        if (several) current.reset_device(first.device());
    }
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
    void* rows(PyObject* o, const char* name, int64_t n, int64_t width, int64_t* ld, at::ScalarType type = at::kBFloat16) const {
        const at::Tensor& t = tensor(o, name);
        check(t, name, type, {n, width});
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

// bf16 or fp32, as the call's first tensor says
bool is_f32(const On& on, const char* name) {
    const auto type = on.first.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) refuse(name, "expected bf16 or fp32");
    return type == at::kFloat;
}

// shape, x, row_of, out, stream -> xs
PyObject* dispatch_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject* {
        const auto s = shape_at<moe_dispatch_shape_t>(v[0]);
        const On on(v[1], "x");
        const bool f32 = is_f32(on, "x");
        const auto type = on.first.scalar_type();
        int64_t ldx;
        const void* x = on.rows(v[1], "x", s.T, s.d, &ldx, type);
        const void* row_of = on.dense(v[2], "row_of", at::kInt, {s.T, s.k});
        const at::Tensor out = on.output(v[3], "out", type, {s.rows, s.d});
        void* const stream = stream_of(v[4]);
        const int rc = call([&] { return p_dispatch_forward(&s, x, ldx, f32, (const int32_t*)row_of, out.data_ptr(), stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped(out);
    });
}

// shape, rows, row_of, weights, out, stream -> tokens (weights None: ones, dispatch's gradient)
PyObject* combine_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 6, [&]() -> PyObject* {
        const auto s = shape_at<moe_dispatch_shape_t>(v[0]);
        const On on(v[1], "rows");
        const bool f32 = is_f32(on, "rows");
        const auto type = on.first.scalar_type();
        const void* rows = on.dense(v[1], "rows", type, {s.rows, s.d});
        const void* row_of = on.dense(v[2], "row_of", at::kInt, {s.T, s.k});
        const void* w = on.optional(v[3], "weights", at::kFloat, {s.T, s.k});
        const at::Tensor out = on.output(v[4], "out", type, {s.T, s.d});
        void* const stream = stream_of(v[5]);
        const int rc = call([&] {
            return w ? p_combine_forward(&s, rows, f32, (const int32_t*)row_of, (const float*)w, out.data_ptr(), stream)
                     : p_dispatch_backward(&s, rows, f32, (const int32_t*)row_of, out.data_ptr(), stream);
        });
        return rc != MOE_OK ? code_of(rc) : wrapped(out);
    });
}

// shape, dy, o, row_of, weights, do, dw, want dw, stream -> (do, dw or None)
PyObject* combine_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject* {
        const auto s = shape_at<moe_dispatch_shape_t>(v[0]);
        const On on(v[1], "dy");
        const bool f32 = is_f32(on, "dy"), want = v[7] == Py_True;
        const auto type = on.first.scalar_type();
        int64_t lddy;
        const void* dy = on.rows(v[1], "dy", s.T, s.d, &lddy, type);
        const void* o = want ? on.dense(v[2], "o", type, {s.rows, s.d}) : nullptr;
        const void* row_of = on.dense(v[3], "row_of", at::kInt, {s.T, s.k});
        const void* w = on.optional(v[4], "weights", at::kFloat, {s.T, s.k});
        const at::Tensor d_o = on.output(v[5], "do", type, {s.rows, s.d});
        at::Tensor dw;
        if (want) dw = on.output(v[6], "dw", at::kFloat, {s.T, s.k});
        void* const stream = stream_of(v[8]);
        const int rc = call([&] {
            return p_combine_backward(&s, dy, lddy, o, f32, (const int32_t*)row_of, (const float*)w, d_o.data_ptr(), want ? (float*)dw.data_ptr() : nullptr, stream);
        });
        if (rc != MOE_OK) return code_of(rc);
        if (want) return wrapped({d_o, dw});
        PyObject* out = wrapped(d_o);
        PyObject* pair = out ? PyTuple_Pack(2, out, Py_None) : nullptr;
        Py_XDECREF(out);
        return pair;
    });
}

struct Stash {
    moe_routing_t routing = {};
    void* saved;
    int64_t rows;
    // offsets, saved; at_h: where the stash's h begins
    Stash(const On& on, const moe_shape_t& s, size_t at_h, PyObject* const* v) {
        rows = (int64_t)s.T * s.k;
        routing.offsets = (const int32_t*)on.dense(v[0], "routing.offsets", at::kInt, {(int64_t)s.e_count + 1});
        const at::Tensor& t = tensor(v[1], "saved");
        on.here(t, "saved");
        if (t.scalar_type() != at::kByte || !t.is_contiguous() || t.numel() < (int64_t)at_h + rows * 2 * s.I) refuse("saved", "expected a stash of this shape");
        saved = t.data_ptr();
    }
};

// shape, saved -> bf16 views of gu [A,2I], h [A,I], o [A,d] in the stash's bytes, A = T k; None where they do not fit
PyObject* saved_views(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 2, [&]() -> PyObject* {
        const auto s = shape_at<moe_shape_t>(v[0]);
        const at::Tensor& t = tensor(v[1], "saved");
        size_t at[3];
        const int rc = p_saved_layout(&s, at, at + 1, at + 2);
        if (rc != MOE_OK) return code_of(rc);
        const int64_t rows = (int64_t)s.T * s.k, cols[3] = {2 * (int64_t)s.I, s.I, s.d};
        if (t.scalar_type() != at::kByte || t.dim() != 1 || !t.is_contiguous() || t.numel() % 2 != 0 || t.storage_offset() % 2 != 0 ||
            t.numel() < (int64_t)at[2] + rows * cols[2] * 2)
            Py_RETURN_NONE;
        const at::Tensor flat = t.view(at::kBFloat16);
        auto view = [&](int i) { return flat.as_strided({rows, cols[i]}, {cols[i], 1}, flat.storage_offset() + (int64_t)at[i] / 2); };
        return wrapped({view(0), view(1), view(2)});
    });
}

// shape, offsets, saved, codes, scales, stream -> (codes, scales)
PyObject* saved_pack(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 6, [&]() -> PyObject* {
        const auto s = shape_at<moe_shape_t>(v[0]);
        const On on(v[2], "saved");
        size_t at_h;
        int rc = p_saved_layout(&s, nullptr, &at_h, nullptr);
        if (rc != MOE_OK) return code_of(rc);
        const Stash in(on, s, at_h, v + 1);
        const at::Tensor codes = on.output(v[3], "codes", at::kChar, {in.rows, 2 * (int64_t)s.I});
        const at::Tensor scales = on.output(v[4], "scales", at::kByte, {in.rows, (int64_t)s.I / 16});
        void* const stream = stream_of(v[5]);
        rc = call([&] { return p_saved_pack(&s, &in.routing, in.saved, codes.data_ptr(), scales.data_ptr(), stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped({codes, scales});
    });
}

// shape, offsets, saved, codes, scales, stream -> None
PyObject* saved_unpack(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 6, [&]() -> PyObject* {
        const auto s = shape_at<moe_shape_t>(v[0]);
        const On on(v[2], "saved");
        size_t at_h;
        int rc = p_saved_layout(&s, nullptr, &at_h, nullptr);
        if (rc != MOE_OK) return code_of(rc);
        const Stash out(on, s, at_h, v + 1);
        const void* codes = on.dense(v[3], "codes", at::kChar, {out.rows, 2 * (int64_t)s.I});
        const void* scales = on.dense(v[4], "scales", at::kByte, {out.rows, (int64_t)s.I / 16});
        void* const stream = stream_of(v[5]);
        rc = call([&] { return p_saved_unpack(&s, &out.routing, codes, scales, out.saved, stream); });
        if (rc != MOE_OK) return code_of(rc);
        Py_RETURN_NONE;
    });
}

int64_t padded(int64_t K) { return (K + 127) / 128 * 128; }

// x, codes, scales, stream -> (codes, scales)
PyObject* mx_quantize(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject* {
        const On on(v[0], "x");
        const bool f32 = is_f32(on, "x");
        if (on.first.dim() != 2) refuse("x", "expected rows");
        const int64_t rows = on.first.size(0), K = on.first.size(1);
        int64_t ldx;
        const void* x = on.rows(v[0], "x", rows, K, &ldx, on.first.scalar_type());
        if (K < 1 || K > 1 << 16) return code_of(MOE_ERR_SHAPE);
        const at::Tensor codes = on.output(v[1], "codes", at::kByte, {rows, padded(K) / 2}), scales = on.output(v[2], "scales", at::kByte, {rows, padded(K) / 32});
        void* const stream = stream_of(v[3]);
        const int rc = call([&] { return p_mx_quantize(x, ldx, f32, rows, (int32_t)K, codes.data_ptr(), scales.data_ptr(), stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped({codes, scales});
    });
}

// w, codes, scales, stream -> (codes, scales)
PyObject* mx_quantize_weights(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject* {
        const On on(v[0], "w");
        if (on.first.dim() != 3) refuse("w", "expected [experts, K, N]");
        const int64_t E = on.first.size(0), K = on.first.size(1), N = on.first.size(2);
        const void* w = on.dense(v[0], "w", at::kBFloat16, {E, K, N});
        if (E < 1 || E > 1 << 16 || K < 1 || K > 1 << 16 || N < 1 || N > 1 << 16) return code_of(MOE_ERR_SHAPE);
        const at::Tensor codes = on.output(v[1], "codes", at::kByte, {E, N, padded(K) / 2}), scales = on.output(v[2], "scales", at::kByte, {E, N, padded(K) / 32});
        void* const stream = stream_of(v[3]);
        const int rc = call([&] { return p_mx_quantize_weights(w, (int32_t)E, (int32_t)K, (int32_t)N, codes.data_ptr(), scales.data_ptr(), stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped({codes, scales});
    });
}

// Sizes of codes and scales [..., K] but for the last
std::vector<int64_t> leading(const On& on, PyObject* scales, int64_t K) {
    const at::Tensor &c = on.first, &s = tensor(scales, "scales");
    on.here(s, "scales");
    if (c.scalar_type() != at::kByte || s.scalar_type() != at::kByte) refuse("codes", "expected bytes");
    if (!c.is_contiguous() || !s.is_contiguous()) refuse("codes", "expected contiguous tensors");
    if (K < 1 || c.dim() < 2 || c.dim() != s.dim() || c.size(-1) != padded(K) / 2 || s.size(-1) != padded(K) / 32) refuse("codes", "sizes");
    std::vector<int64_t> sizes(c.sizes().begin(), c.sizes().end() - 1);
    for (size_t i = 0; i < sizes.size(); ++i)
        if (s.size((int64_t)i) != sizes[i]) refuse("scales", "sizes");
    return sizes;
}

// codes, scales, K, fp32, out, stream -> values
PyObject* mx_values(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 6, [&]() -> PyObject* {
        const On on(v[0], "codes");
        const int64_t K = PyLong_AsLongLong(v[2]);
        if (PyErr_Occurred()) return nullptr;
        if (K < 1 || K > 1 << 16) return code_of(MOE_ERR_SHAPE);
        std::vector<int64_t> sizes = leading(on, v[1], K);
        int64_t rows = 1;
        for (int64_t m : sizes) rows *= m;
        sizes.push_back(K);
        const bool f32 = v[3] == Py_True;
        const auto type = f32 ? at::kFloat : at::kBFloat16;
        at::Tensor out;
        if (v[4] == Py_None) {
            out = made(on.first, type, sizes);
        } else {
            out = tensor(v[4], "out");
            on.here(out, "out");
            if (out.scalar_type() != type) refuse("out", "type");
            if (out.sizes() != at::IntArrayRef(sizes) || !out.is_contiguous()) refuse("out", "sizes");
        }
        void* const stream = stream_of(v[5]);
        const void *codes = on.first.data_ptr(), *scales = tensor(v[1], "scales").data_ptr();
        const int rc = call([&] { return p_mx_values(codes, scales, rows, (int32_t)K, out.data_ptr(), f32, stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped(out);
    });
}

struct MxOperand {
    void *codes, *scales;
    // codes and scales of `sizes` rows, of K values each
    MxOperand(const On& on, PyObject* const* v, std::initializer_list<int64_t> sizes, int64_t K) {
        std::vector<int64_t> c(sizes), s(sizes);
        c.push_back(padded(K) / 2), s.push_back(padded(K) / 32);
        codes = checked(on, v[0], "codes", c);
        scales = checked(on, v[1], "scales", s);
    }
    static void* checked(const On& on, PyObject* o, const char* name, const std::vector<int64_t>& sizes) {
        const at::Tensor& t = tensor(o, name);
        on.here(t, name);
        if (t.scalar_type() != at::kByte) refuse(name, "type");
        if (t.sizes() != at::IntArrayRef(sizes)) refuse(name, "sizes");
        if (!t.is_contiguous()) refuse(name, "expected a contiguous tensor");
        return t.data_ptr();
    }
};
int32_t whole(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (PyErr_Occurred()) throw Refused{};
    return v < INT32_MIN || v > INT32_MAX ? 0 : (int32_t)v;
}

// shape, a's codes and scales, w's, offsets, perm, k, fp32, y, stream -> y
PyObject* mx_product(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 11, [&]() -> PyObject* {
        const auto s = shape_at<moe_mx_shape_t>(v[0]);
        const On on(v[1], "codes");
        const int64_t a_rows = on.first.dim() > 0 ? on.first.size(0) : 0;
        const MxOperand a(on, v + 1, {a_rows}, s.K), w(on, v + 3, {s.experts, s.N}, s.K);
        const int32_t* offsets = (const int32_t*)on.dense(v[5], "offsets", at::kInt, {(int64_t)s.experts + 1});
        const int32_t* perm = (const int32_t*)on.optional(v[6], "perm", at::kInt, {s.rows});
        const int32_t k = whole(v[7]);
        const bool f32 = v[8] == Py_True;
        const at::Tensor y = on.output(v[9], "y", f32 ? at::kFloat : at::kBFloat16, {s.rows, s.N});
        void* const stream = stream_of(v[10]);
        void* const out = y.data_ptr();
        const int rc = call([&] { return p_mx_product(&s, a.codes, a.scales, a_rows, perm, k, w.codes, w.scales, offsets, out, f32, stream); });
        return rc != MOE_OK ? code_of(rc) : wrapped(y);
    });
}

// shape, a's codes and scales, the gate's, up's, offsets, perm, k, quantize, h or codes, scales, stream -> h or (codes, scales)
PyObject* mx_gate_up(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 14, [&]() -> PyObject* {
        const auto s = shape_at<moe_mx_shape_t>(v[0]);
        const On on(v[1], "codes");
        const int64_t a_rows = on.first.dim() > 0 ? on.first.size(0) : 0;
        const MxOperand a(on, v + 1, {a_rows}, s.K), g(on, v + 3, {s.experts, s.N}, s.K), u(on, v + 5, {s.experts, s.N}, s.K);
        const int32_t* offsets = (const int32_t*)on.dense(v[7], "offsets", at::kInt, {(int64_t)s.experts + 1});
        const int32_t* perm = (const int32_t*)on.optional(v[8], "perm", at::kInt, {s.rows});
        const int32_t k = whole(v[9]);
        const bool quantize = v[10] == Py_True;
        at::Tensor h, scales;
        if (quantize) {
            h = on.output(v[11], "h codes", at::kByte, {s.rows, padded(s.N) / 2});
            scales = on.output(v[12], "h scales", at::kByte, {s.rows, padded(s.N) / 32});
        } else {
            h = on.output(v[11], "h", at::kBFloat16, {s.rows, s.N});
        }
        void* const stream = stream_of(v[13]);
        void *const out = h.data_ptr(), *const out_scales = quantize ? scales.data_ptr() : nullptr;
        const int rc = call([&] {
            return p_mx_gate_up(&s, a.codes, a.scales, a_rows, perm, k, g.codes, g.scales, u.codes, u.scales, offsets, quantize ? nullptr : out, quantize ? out : nullptr,
                                out_scales, stream);
        });
        if (rc != MOE_OK) return code_of(rc);
        return quantize ? wrapped({h, scales}) : wrapped(h);
    });
}

// addresses of the library's functions, in the order of the pointers above
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded(n, 19, [&]() -> PyObject* {
        void* f[19];
        for (int i = 0; i < 19; ++i) f[i] = stream_of(v[i]);
        int i = 0;
        auto take = [&](auto& p) { p = (std::decay_t<decltype(p)>)f[i++]; };
        take(p_adapter_plan), take(p_adapter_forward), take(p_adapter_backward), take(p_balance_forward), take(p_balance_backward), take(p_adapter_bytes);
        take(p_balance_bytes), take(p_dispatch_forward), take(p_dispatch_backward), take(p_combine_forward), take(p_combine_backward), take(p_saved_pack);
        take(p_saved_unpack), take(p_mx_quantize), take(p_mx_quantize_weights), take(p_mx_values);
        take(p_mx_product), take(p_mx_gate_up), take(p_saved_layout);
        Py_RETURN_NONE;
    });
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(adapter_plan), FAST(adapter_forward), FAST(adapter_backward), FAST(balance_forward), FAST(balance_backward), FAST(dispatch_forward),
                         FAST(combine_forward), FAST(combine_backward), FAST(saved_pack), FAST(saved_unpack), FAST(mx_quantize), FAST(mx_quantize_weights),
                         FAST(mx_values), FAST(mx_product), FAST(mx_gate_up), FAST(saved_views), FAST(bind),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() { return PyModule_Create(&module); }
