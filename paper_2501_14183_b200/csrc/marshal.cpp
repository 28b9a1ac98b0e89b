// Python's way into the C ABI: takes tensors and configuration structs as the binding's functions get them and calls the library.
//
// The host side of a small step is its longest part (four calls of 4.6 to 6.2 us where a launch is about 2): marshalling thirty pointers
// through ctypes and Python attribute calls costs more than half as much again as the launches.  Here a pointer is read from the tensor
// object itself and the stream from PyTorch's current one.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <vector>

#include "../../include/vardrop.h"

namespace {

// The arguments of one call; the first problem leaves a Python exception set and `ok` false.
struct Args {
    PyObject* const* a;
    bool ok = true;
    Py_buffer cfg_view{};
    bool has_cfg = false;

    explicit Args(PyObject* const* args) : a(args) {}
    ~Args() { if (has_cfg) PyBuffer_Release(&cfg_view); }

    // device address of a tensor (or of anything with a data_ptr method); None: NULL
    template <typename T = void>
    T* ptr(int i) {
        PyObject* t = a[i];
        if (!ok || t == Py_None) return nullptr;
        if (THPVariable_Check(t)) return static_cast<T*>(THPVariable_Unpack(t).data_ptr());
        PyObject* v = PyObject_CallMethod(t, "data_ptr", nullptr);
        void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
        Py_XDECREF(v);
        ok = !PyErr_Occurred();
        return static_cast<T*>(p);
    }
    // The same for the operators around the attention, whose tensors come from many places: on the current device, contiguous (`kStrided`: with strides that the
    // configuration gives; `kDense`: in any order of its dimensions), of the type, and with at least so many elements.  None: NULL.
    enum Layout { kContiguous, kDense, kStrided };
    template <typename T = void>
    T* checked(int i, const char* name, at::ScalarType type, int64_t count, Layout layout = kContiguous) {
        if (!ok || a[i] == Py_None) return nullptr;
        if (!THPVariable_Check(a[i])) return refuse<T>("%s is not a tensor", name);
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda()) return refuse<T>("%s is not a CUDA tensor", name);
        if (t.get_device() != c10::cuda::current_device()) return refuse<T>("%s is on another device than the current one", name);
        if (t.scalar_type() != type) return refuse<T>("%s has another type than the call expects", name);
        if (layout == kContiguous ? !t.is_contiguous() : layout == kDense && !t.is_non_overlapping_and_dense()) return refuse<T>("%s is not contiguous", name);
        if (t.numel() < count) return refuse<T>("%s has fewer elements than the configuration says", name);
        return static_cast<T*>(t.data_ptr());
    }
    // q, k or v of a packed call: [T, H, D] with the strides of the configuration
    const void* packed(int i, const char* name, const vardrop_packed_cfg& c, int H, int64_t sT, int64_t sH) {
        const bool plain = sT == 0 && sH == 0;
        void* const p = checked(i, name, at::kBFloat16, static_cast<int64_t>(c.T) * H * c.D, plain ? kContiguous : kStrided);
        if (!p || plain) return p;
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (t.dim() != 3 || t.size(0) != c.T || t.size(1) != H || t.size(2) != c.D || (c.T > 1 && t.stride(0) != sT) || (H > 1 && t.stride(1) != sH) || t.stride(2) != 1)
            return refuse<void>("%s does not have the shape and strides of the configuration", name);
        return p;
    }
    // a branch of an activation: [B, N, C] with the row stride of the configuration
    void* branch(int i, const char* name, const vardrop_act_cfg& c, at::ScalarType type) {
        void* const p = checked(i, name, type, static_cast<int64_t>(c.B) * c.N * c.C, c.stride == 0 ? kContiguous : kStrided);
        if (!p || c.stride == 0) return p;
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (t.dim() != 3 || t.size(0) != c.B || t.size(1) != c.N || t.size(2) != c.C || (c.N > 1 && t.stride(1) != c.stride) || (c.B > 1 && t.stride(0) != c.N * c.stride) ||
            (c.C > 1 && t.stride(2) != 1))
            return refuse<void>("%s does not have the shape and strides of the configuration", name);
        return p;
    }
    template <typename T>
    T* refuse(const char* text, const char* name) {
        PyErr_Format(PyExc_ValueError, text, name);
        ok = false;
        return nullptr;
    }
    // a ctypes struct through the buffer protocol
    template <typename T>
    const T* cfg(int i) {
        if (!ok) return nullptr;
        has_cfg = PyObject_GetBuffer(a[i], &cfg_view, PyBUF_SIMPLE) == 0;
        if (has_cfg && cfg_view.len < static_cast<Py_ssize_t>(sizeof(T))) PyErr_SetString(PyExc_TypeError, "configuration struct of another kind");
        ok = !PyErr_Occurred();
        return static_cast<const T*>(cfg_view.buf);
    }
    size_t bytes(int i) {
        if (!ok) return 0;
        if (THPVariable_Check(a[i])) return THPVariable_Unpack(a[i]).nbytes();
        PyObject* n = PyObject_CallMethod(a[i], "numel", nullptr);
        PyObject* e = n ? PyObject_CallMethod(a[i], "element_size", nullptr) : nullptr;
        const size_t r = e ? PyLong_AsSize_t(n) * PyLong_AsSize_t(e) : 0;
        Py_XDECREF(n);
        Py_XDECREF(e);
        ok = !PyErr_Occurred();
        return r;
    }
};

// Runs `call` with PyTorch's current stream and without the interpreter lock; returns its status.
template <typename F>
PyObject* finish(const Args& args, F call) {
    if (!args.ok) return nullptr;
    void* const stream = c10::cuda::getCurrentCUDAStream().stream();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}
template <int kCount, typename F>
PyObject* guarded(PyObject* const* a, Py_ssize_t n, F body) {
    if (n != kCount) return PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", kCount, n);
    try {
        Args args(a);
        return body(args);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject* hash(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<6>(a, n, [](Args& g) {
        const auto x = g.ptr<const float>(0);
        const auto cfg = g.cfg<vardrop_hash_cfg>(1);
        const auto keys = g.ptr<uint64_t>(2);
        const auto freqs = g.ptr<int32_t>(3);
        const auto amp = g.ptr<float>(4);
        const auto ws = g.ptr(5);
        const size_t nb = g.bytes(5);
        return finish(g, [=](void* s) { return vardrop_hash(x, cfg, keys, freqs, amp, ws, nb, s); });
    });
}
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<10>(a, n, [](Args& g) {
        const auto keys = g.ptr<const uint64_t>(0);
        const auto cfg = g.cfg<vardrop_select_cfg>(1);
        int32_t* o[7];
        for (int i = 0; i < 7; ++i) o[i] = g.ptr<int32_t>(2 + i);
        const auto ws = g.ptr(9);
        const size_t nb = g.bytes(9);
        return finish(g, [=](void* s) { return vardrop_select(keys, cfg, o[0], o[1], o[2], o[3], o[4], o[5], o[6], ws, nb, s); });
    });
}
PyObject* select_static(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<9>(a, n, [](Args& g) {
        const auto keys = g.ptr<const uint64_t>(0);
        const auto cfg = g.cfg<vardrop_select_cfg>(1);
        int32_t* o[7];
        for (int i = 0; i < 7; ++i) o[i] = g.ptr<int32_t>(2 + i);
        return finish(g, [=](void* s) { return vardrop_select_static(keys, cfg, o[0], o[1], o[2], o[3], o[4], o[5], o[6], s); });
    });
}
PyObject* gather_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<5>(a, n, [](Args& g) {
        const auto x = g.ptr<const float>(0);
        const auto sel = g.ptr<const int32_t>(1), n_sel = g.ptr<const int32_t>(2);
        const auto cfg = g.cfg<vardrop_gather_cfg>(3);
        const auto out = g.ptr<float>(4);
        return finish(g, [=](void* s) { return vardrop_gather_rows(x, sel, n_sel, cfg, out, s); });
    });
}
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<9>(a, n, [](Args& g) {
        const void* const q = g.ptr(0);
        const void* const k = g.ptr(1);
        const void* const v = g.ptr(2);
        const auto sel = g.ptr<const int32_t>(3), n_sel = g.ptr<const int32_t>(4);
        const auto cfg = g.cfg<vardrop_attn_cfg>(5);
        const auto o = g.ptr(6);
        const auto lse = g.ptr<float>(7);
        const auto ws = g.ptr(8);
        const size_t nb = g.bytes(8);
        return finish(g, [=](void* s) { return vardrop_attn_fwd(q, k, v, sel, n_sel, cfg, o, lse, ws, nb, s); });
    });
}
PyObject* attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<14>(a, n, [](Args& g) {
        const void* const q = g.ptr(0);
        const void* const k = g.ptr(1);
        const void* const v = g.ptr(2);
        const void* const o = g.ptr(3);
        const auto lse = g.ptr<const float>(4);
        const void* const d_o = g.ptr(5);
        const auto sel = g.ptr<const int32_t>(6), n_sel = g.ptr<const int32_t>(7), inv = g.ptr<const int32_t>(8);
        const auto cfg = g.cfg<vardrop_attn_cfg>(9);
        const auto dq = g.ptr(10), dk = g.ptr(11), dv = g.ptr(12), ws = g.ptr(13);
        const size_t nb = g.bytes(13);
        return finish(g, [=](void* s) { return vardrop_attn_bwd(q, k, v, o, lse, d_o, sel, n_sel, inv, cfg, dq, dk, dv, ws, nb, s); });
    });
}
PyObject* pearson_max(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<5>(a, n, [](Args& g) {
        const auto x = g.ptr<const float>(0);
        const auto cfg = g.cfg<vardrop_pearson_cfg>(1);
        const auto rho = g.ptr<float>(2);
        const auto above = g.ptr<int32_t>(3);
        const auto ws = g.ptr(4);
        const size_t nb = g.bytes(4);
        return finish(g, [=](void* s) { return vardrop_pearson_max(x, cfg, rho, above, ws, nb, s); });
    });
}

PyObject* packed_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<3>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_packed_cfg>(1);
        if (!g.ok) return nullptr;
        const auto cu = g.checked<const int32_t>(0, "cu_seqlens", at::kInt, static_cast<int64_t>(cfg->n_seqs) + 1);
        void* const plan = g.checked(2, "plan", at::kByte, 0);
        const size_t nb = g.ok && plan ? g.bytes(2) : 0;
        return finish(g, [=](void* s) { return vardrop_packed_plan(cu, cfg, plan, nb, s); });
    });
}
PyObject* attn_packed_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<8>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_packed_cfg>(4);
        if (!g.ok) return nullptr;
        const int64_t rows = static_cast<int64_t>(cfg->T) * cfg->Hq;
        const void* const q = g.packed(0, "q", *cfg, cfg->Hq, cfg->sTq, cfg->sHq);
        const void* const k = g.packed(1, "k", *cfg, cfg->Hkv, cfg->sTkv, cfg->sHkv);
        const void* const v = g.packed(2, "v", *cfg, cfg->Hkv, cfg->sTkv, cfg->sHkv);
        const void* const plan = g.checked(3, "plan", at::kByte, 0);
        const size_t np = g.ok && plan ? g.bytes(3) : 0;
        void* const o = g.checked(5, "o", at::kBFloat16, rows * cfg->D);
        const auto lse = g.checked<float>(6, "lse", at::kFloat, rows);
        void* const ws = g.checked(7, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(7) : 0;
        return finish(g, [=](void* s) { return vardrop_attn_packed_fwd(q, k, v, plan, np, cfg, o, lse, ws, nb, s); });
    });
}
PyObject* attn_packed_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<12>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_packed_cfg>(7);
        if (!g.ok) return nullptr;
        const int64_t rows = static_cast<int64_t>(cfg->T) * cfg->Hq, kv = static_cast<int64_t>(cfg->T) * cfg->Hkv * cfg->D;
        const void* const q = g.packed(0, "q", *cfg, cfg->Hq, cfg->sTq, cfg->sHq);
        const void* const k = g.packed(1, "k", *cfg, cfg->Hkv, cfg->sTkv, cfg->sHkv);
        const void* const v = g.packed(2, "v", *cfg, cfg->Hkv, cfg->sTkv, cfg->sHkv);
        const void* const o = g.checked(3, "o", at::kBFloat16, rows * cfg->D);
        const auto lse = g.checked<const float>(4, "lse", at::kFloat, rows);
        const void* const d_o = g.checked(5, "d_o", at::kBFloat16, rows * cfg->D);
        const void* const plan = g.checked(6, "plan", at::kByte, 0);
        const size_t np = g.ok && plan ? g.bytes(6) : 0;
        void* const dq = g.checked(8, "dq", at::kBFloat16, rows * cfg->D);
        void* const dk = g.checked(9, "dk", at::kBFloat16, kv);
        void* const dv = g.checked(10, "dv", at::kBFloat16, kv);
        void* const ws = g.checked(11, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(11) : 0;
        return finish(g, [=](void* s) { return vardrop_attn_packed_bwd(q, k, v, o, lse, d_o, plan, np, cfg, dq, dk, dv, ws, nb, s); });
    });
}

at::ScalarType type_of(int dtype) { return dtype == 2 ? at::kFloat : dtype == 1 ? at::kHalf : at::kBFloat16; }

PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<13>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_norm_cfg>(9);
        if (!g.ok) return nullptr;
        const at::ScalarType ty = type_of(cfg->dtype);
        const int64_t C = cfg->C, rows = static_cast<int64_t>(cfg->B) * cfg->N, all = rows * C, S = cfg->S > 1 ? cfg->S : 1;
        const void* const x = g.checked(0, "x", ty, all);
        const void* const y = g.checked(1, "y", ty, all);
        const auto gate = g.checked<const float>(2, "gate", at::kFloat, cfg->gate_rows * C);
        const auto w_post = g.checked<const float>(3, "w_post", at::kFloat, C), b_post = g.checked<const float>(4, "b_post", at::kFloat, C);
        const auto w_pre = g.checked<const float>(5, "w_pre", at::kFloat, C), b_pre = g.checked<const float>(6, "b_pre", at::kFloat, C);
        const auto sel = g.checked<const int32_t>(7, "sel_idx", at::kInt, S * cfg->N), n_sel = g.checked<const int32_t>(8, "n_sel", at::kInt, S);
        void* const h = g.checked(10, "h", ty, all);
        void* const u = g.checked(11, "u", ty, all);
        const auto stats = g.checked<float>(12, "stats", at::kFloat, rows * 4);
        return finish(g, [=](void* s) { return vardrop_norm_fwd(x, y, gate, w_post, b_post, w_pre, b_pre, sel, n_sel, cfg, h, u, stats, s); });
    });
}
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<21>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_norm_cfg>(12);
        if (!g.ok) return nullptr;
        const at::ScalarType ty = type_of(cfg->dtype);
        const int64_t C = cfg->C, rows = static_cast<int64_t>(cfg->B) * cfg->N, all = rows * C, S = cfg->S > 1 ? cfg->S : 1;
        const void* const x = g.checked(0, "x", ty, all);
        const void* const y = g.checked(1, "y", ty, all);
        const auto gate = g.checked<const float>(2, "gate", at::kFloat, cfg->gate_rows * C);
        const auto w_post = g.checked<const float>(3, "w_post", at::kFloat, C), b_post = g.checked<const float>(4, "b_post", at::kFloat, C);
        const auto w_pre = g.checked<const float>(5, "w_pre", at::kFloat, C);
        const auto sel = g.checked<const int32_t>(6, "sel_idx", at::kInt, S * cfg->N), n_sel = g.checked<const int32_t>(7, "n_sel", at::kInt, S);
        const auto inv = g.checked<const int32_t>(8, "inv_idx", at::kInt, S * cfg->N);
        const auto stats = g.checked<const float>(9, "stats", at::kFloat, rows * 4);
        const void* const d_h = g.checked(10, "d_h", ty, all);
        const void* const d_u = g.checked(11, "d_u", ty, all);
        void* const dx = g.checked(13, "dx", ty, all);
        void* const dy = g.checked(14, "dy", ty, all);
        const auto d_gate = g.checked<float>(15, "d_gate", at::kFloat, cfg->gate_rows * C);
        const auto d_w_post = g.checked<float>(16, "d_w_post", at::kFloat, C), d_b_post = g.checked<float>(17, "d_b_post", at::kFloat, C);
        const auto d_w_pre = g.checked<float>(18, "d_w_pre", at::kFloat, C), d_b_pre = g.checked<float>(19, "d_b_pre", at::kFloat, C);
        void* const ws = g.checked(20, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(20) : 0;
        return finish(g, [=](void* s) {
            return vardrop_norm_bwd(x, y, gate, w_post, b_post, w_pre, sel, n_sel, inv, stats, d_h, d_u, cfg, dx, dy, d_gate, d_w_post, d_b_post, d_w_pre, d_b_pre, ws, nb, s);
        });
    });
}
// the tensors of a list or tuple; `out` None: in place
PyObject* grad_clip(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<5>(a, n, [&](Args& g) -> PyObject* {
        PyObject* const in = a[0];
        PyObject* const out = a[2];
        const bool same = out == Py_None;
        if (!(PyList_Check(in) || PyTuple_Check(in)) || !(same || PyList_Check(out) || PyTuple_Check(out)))
            return PyErr_Format(PyExc_TypeError, "grads has to be a list or tuple of tensors, outs one or None");
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(in);
        if (!same && PySequence_Fast_GET_SIZE(out) != count) return PyErr_Format(PyExc_ValueError, "%zd tensors and %zd outputs", count, PySequence_Fast_GET_SIZE(out));
        std::vector<vardrop_tensor> table(static_cast<size_t>(count));
        Args ins(PySequence_Fast_ITEMS(in)), outs(same ? PySequence_Fast_ITEMS(in) : PySequence_Fast_ITEMS(out));
        for (Py_ssize_t i = 0; i < count; ++i) {
            if (!THPVariable_Check(ins.a[i])) return PyErr_Format(PyExc_ValueError, "a gradient is not a tensor");
            const at::Tensor& t = THPVariable_Unpack(ins.a[i]);
            const at::ScalarType ty = t.scalar_type();
            vardrop_tensor& e = table[static_cast<size_t>(i)];
            if (ty != at::kBFloat16 && ty != at::kHalf && ty != at::kFloat) return PyErr_Format(PyExc_ValueError, "a gradient is neither bf16, fp16 nor fp32");
            e.in = ins.checked(static_cast<int>(i), "a gradient", ty, 0, Args::kDense);
            e.n = t.numel();
            e.out = same ? const_cast<void*>(e.in) : outs.checked(static_cast<int>(i), "an output", ty, e.n, Args::kDense);
            e.dtype = ty == at::kFloat ? 2 : ty == at::kHalf ? 1 : 0;
            e.reserved = 0;
            if (!ins.ok || !outs.ok) return nullptr;
            if (same) continue;
            if (!THPVariable_Check(outs.a[i])) return PyErr_Format(PyExc_ValueError, "an output is not a tensor");
            const at::Tensor& o = THPVariable_Unpack(outs.a[i]);
            if (o.sizes() != t.sizes() || o.strides() != t.strides()) return PyErr_Format(PyExc_ValueError, "an output has another shape or other strides than its gradient");
        }
        const auto cfg = g.cfg<vardrop_clip_cfg>(1);
        const auto norm = g.checked<float>(3, "norm", at::kFloat, 1);
        void* const ws = g.checked(4, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(4) : 0;
        const vardrop_tensor* const tensors = table.data();
        return finish(g, [=](void* s) { return vardrop_grad_clip(tensors, static_cast<int32_t>(count), cfg, norm, ws, nb, s); });
    });
}
PyObject* embed_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<5>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_embed_cfg>(2);
        if (!g.ok) return nullptr;
        const int64_t T = cfg->T, V = cfg->V, C = cfg->C;
        const void* const table = g.checked(0, "table", type_of(cfg->dtype), V * C);
        const auto idx = g.checked<const int32_t>(1, "idx", at::kInt, T);
        void* const out = g.checked(3, "out", type_of(cfg->out_dtype), T * C);
        void* const ws = g.checked(4, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(4) : 0;
        return finish(g, [=](void* s) { return vardrop_embed_fwd(table, idx, cfg, out, ws, nb, s); });
    });
}
PyObject* embed_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<5>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_embed_cfg>(2);
        if (!g.ok) return nullptr;
        const int64_t T = cfg->T, V = cfg->V, C = cfg->C;
        const void* const d_out = g.checked(0, "d_out", type_of(cfg->out_dtype), T * C);
        const auto idx = g.checked<const int32_t>(1, "idx", at::kInt, T);
        void* const d_table = g.checked(3, "d_table", type_of(cfg->dtype), V * C);
        void* const ws = g.checked(4, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(4) : 0;
        return finish(g, [=](void* s) { return vardrop_embed_bwd(d_out, idx, cfg, d_table, ws, nb, s); });
    });
}
PyObject* act_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<6>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_act_cfg>(3);
        if (!g.ok) return nullptr;
        const at::ScalarType ty = type_of(cfg->dtype);
        const void* const in = g.branch(0, "a", *cfg, ty);
        const void* const gate = g.branch(1, "b", *cfg, ty);
        const auto n_sel = g.checked<const int32_t>(2, "n_sel", at::kInt, cfg->S > 1 ? cfg->S : 1);
        void* const y = g.checked(4, "y", ty, static_cast<int64_t>(cfg->B) * cfg->N * cfg->C);
        void* const ckpt = g.checked(5, "ckpt", at::kByte, 0);
        const size_t nb = g.ok && ckpt ? g.bytes(5) : 0;
        return finish(g, [=](void* s) { return vardrop_act_fwd(in, gate, n_sel, cfg, y, ckpt, nb, s); });
    });
}
PyObject* act_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<7>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_act_cfg>(3);
        if (!g.ok) return nullptr;
        const at::ScalarType ty = type_of(cfg->dtype);
        const int64_t all = static_cast<int64_t>(cfg->B) * cfg->N * cfg->C;
        const void* const d_y = g.checked(0, "d_y", ty, all);
        const void* const ckpt = g.checked(1, "ckpt", at::kByte, 0);
        const auto n_sel = g.checked<const int32_t>(2, "n_sel", at::kInt, cfg->S > 1 ? cfg->S : 1);
        void* const d_a = g.branch(4, "d_a", *cfg, ty);
        void* const d_b = g.branch(5, "d_b", *cfg, ty);
        void* const y = g.checked(6, "y", ty, all);
        const size_t nb = g.ok && ckpt ? g.bytes(1) : 0;
        return finish(g, [=](void* s) { return vardrop_act_bwd(d_y, ckpt, nb, n_sel, cfg, d_a, d_b, y, s); });
    });
}
PyObject* loss_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<7>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_loss_cfg>(3);
        if (!g.ok) return nullptr;
        const at::ScalarType ty = type_of(cfg->dtype);
        const int64_t T = cfg->T, V = cfg->V, C = cfg->C;
        const void* const h = g.checked(0, "h", ty, T * C);
        const void* const w = g.checked(1, "w", ty, V * C);
        const auto labels = g.checked<const int32_t>(2, "labels", at::kInt, T);
        const auto loss = g.checked<float>(4, "loss", at::kFloat, T), lse = g.checked<float>(5, "lse", at::kFloat, T);
        void* const ws = g.checked(6, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(6) : 0;
        return finish(g, [=](void* s) { return vardrop_loss_fwd(h, w, labels, cfg, loss, lse, ws, nb, s); });
    });
}
PyObject* loss_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<9>(a, n, [](Args& g) -> PyObject* {
        const auto cfg = g.cfg<vardrop_loss_cfg>(5);
        if (!g.ok) return nullptr;
        const at::ScalarType ty = type_of(cfg->dtype);
        const int64_t T = cfg->T, V = cfg->V, C = cfg->C;
        const void* const h = g.checked(0, "h", ty, T * C);
        const void* const w = g.checked(1, "w", ty, V * C);
        const auto labels = g.checked<const int32_t>(2, "labels", at::kInt, T);
        const auto lse = g.checked<const float>(3, "lse", at::kFloat, T), d_loss = g.checked<const float>(4, "d_loss", at::kFloat, T);
        void* const d_h = g.checked(6, "d_h", ty, T * C);
        void* const d_w = g.checked(7, "d_w", ty, V * C);
        void* const ws = g.checked(8, "ws", at::kByte, 0);
        const size_t nb = g.ok && ws ? g.bytes(8) : 0;
        return finish(g, [=](void* s) { return vardrop_loss_bwd(h, w, labels, lse, d_loss, cfg, d_h, d_w, ws, nb, s); });
    });
}

#define VD_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {VD_METHOD(hash), VD_METHOD(select), VD_METHOD(select_static), VD_METHOD(gather_rows), VD_METHOD(attn_fwd), VD_METHOD(attn_bwd),
                           VD_METHOD(pearson_max), VD_METHOD(packed_plan), VD_METHOD(attn_packed_fwd), VD_METHOD(attn_packed_bwd), VD_METHOD(norm_fwd), VD_METHOD(norm_bwd), VD_METHOD(grad_clip), VD_METHOD(embed_fwd), VD_METHOD(embed_bwd), VD_METHOD(act_fwd), VD_METHOD(act_bwd),
                           VD_METHOD(loss_fwd), VD_METHOD(loss_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__marshal(void) { return PyModule_Create(&g_module); }
