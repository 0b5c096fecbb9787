// CPython entries, first of all for the call that a decoder makes most, dps_linear: argument checks, output allocation and the current stream
// in native code, then the same C ABI function of libdps.so.  Small layers are bound by the host: a call of a 512 x 512 layer takes 13.0 us through ctypes, 4.6 us through here.
// Anything out of the ordinary (another tensor type, a wrong dtype, a shape that does not fit) returns None, and the caller
// takes the ctypes path, which says what is wrong.  A status other than 0 is returned as an int: the call was made once, and
// is not made again.  The GIL is released around the allocation and the call, as ctypes and PyTorch's operators do: either may
// block (a full launch queue, a first call's set-up), and what they wait for may need Python.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/dps.h"

namespace {

using LinearFn = int (*)(int32_t, int32_t, const void*, const uint8_t*, const uint8_t*, void*, int64_t, int64_t, int64_t, void*);
LinearFn g_linear = nullptr;

struct WithoutGil {
    PyThreadState* state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

// set_linear(address of dps_linear)
PyObject* set_linear(PyObject*, PyObject* arg) {
    g_linear = reinterpret_cast<LinearFn>(PyLong_AsVoidPtr(arg));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

bool plain(const at::Tensor& t, at::ScalarType type) {
    return t.is_cuda() && t.scalar_type() == type && t.layout() == at::kStrided && t.is_contiguous();
}

// linear(mode, enc, x, w_persist, w_resid or None, y or None) -> y, or a status that is not 0, or None: use the other path
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 6 || g_linear == nullptr || !PyLong_Check(args[0]) || !PyLong_Check(args[1])) Py_RETURN_NONE;
    if (!THPVariable_CheckExact(args[2]) || !THPVariable_CheckExact(args[3])) Py_RETURN_NONE;
    if (args[4] != Py_None && !THPVariable_CheckExact(args[4])) Py_RETURN_NONE;
    if (args[5] != Py_None && !THPVariable_CheckExact(args[5])) Py_RETURN_NONE;
    const long mode = PyLong_AsLong(args[0]), enc = PyLong_AsLong(args[1]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (mode < 0 || mode > 1 || enc < 0 || enc > 255) Py_RETURN_NONE;
    try {
        const at::Tensor& x = THPVariable_Unpack(args[2]);
        const at::Tensor& p = THPVariable_Unpack(args[3]);
        if (!plain(x, at::kHalf) || !plain(p, at::kByte) || x.dim() != 2 || p.dim() != 2 || x.size(1) != p.size(1)) Py_RETURN_NONE;
        const uint8_t* r = nullptr;
        if (args[4] != Py_None) {
            const at::Tensor& t = THPVariable_Unpack(args[4]);
            if (!plain(t, at::kByte)) Py_RETURN_NONE;
            r = t.const_data_ptr<uint8_t>();
        }
        const int64_t m = x.size(0), rows = p.size(0), k = x.size(1);
        const void* px = x.const_data_ptr();
        const uint8_t* pp = p.const_data_ptr<uint8_t>();
        PyObject* out = args[5];
        at::Tensor y;
        if (out != Py_None) {
            y = THPVariable_Unpack(out);
            if (!plain(y, at::kHalf)) Py_RETURN_NONE;
        }
        int status = 0;
        {
            const auto device = x.device();
            WithoutGil nogil;   // (the caller's frame holds the argument tensors)
            if (!y.defined()) y = at::empty({m, rows}, at::TensorOptions().dtype(at::kHalf).device(device));
            status = g_linear((int32_t)mode, (int32_t)enc, px, pp, r, y.mutable_data_ptr(), m, rows, k,
                              c10::cuda::getCurrentCUDAStream().stream());
        }
        if (status != 0) return PyLong_FromLong(status);
        if (out != Py_None) {
            Py_INCREF(out);
            return out;
        }
        return THPVariable_Wrap(y);
    } catch (...) {     // out of memory, an exotic tensor: the other path meets it again and reports it
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// ---- the calls that load a model and serve experts --------------------------------------------------------------------
// A loader waits for the answer of an AUTO split before it can go on, and the GPU waits with it: a layer of four tensors, split
// and rebuilt, takes 291 us through here, 309 through ctypes; two grouped calls occupy the host for 15-25 us instead of 35-46.

struct Functions {
    int (*split)(const void*, uint8_t*, uint8_t*, int64_t, int64_t, int32_t*, void*) = nullptr;
    int (*reconstruct)(const uint8_t*, const uint8_t*, void*, int64_t, int64_t, int32_t, void*) = nullptr;
    int (*moe)(int32_t, const int32_t*, const void*, const int32_t*, const int32_t*, const uint8_t*, const uint8_t*, void*, int64_t,
               int64_t, int64_t, int64_t, int32_t, void*, size_t, void*) = nullptr;
} g_fn;

// set_functions(addresses of dps_split_weights, dps_reconstruct, dps_moe_linear)
PyObject* set_functions(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "three addresses");
        return nullptr;
    }
    void* at[3];
    for (int i = 0; i < 3; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_fn.split = reinterpret_cast<decltype(g_fn.split)>(at[0]);
    g_fn.reconstruct = reinterpret_cast<decltype(g_fn.reconstruct)>(at[1]);
    g_fn.moe = reinterpret_cast<decltype(g_fn.moe)>(at[2]);
    Py_RETURN_NONE;
}

// A plain CUDA tensor of this type, `dims` dimensions (0: any) in `arg`.  None leaves `out` undefined if `optional`.
bool take(PyObject* arg, at::ScalarType type, int dims, bool optional, at::Tensor& out) {
    if (arg == Py_None) return optional;
    if (!THPVariable_CheckExact(arg)) return false;
    out = THPVariable_Unpack(arg);
    return plain(out, type) && (dims == 0 || out.dim() == dims);
}
bool small_int(PyObject* arg, int32_t& out) {
    if (!PyLong_Check(arg)) return false;
    const long v = PyLong_AsLong(arg);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    out = (int32_t)v;
    return v >= 0 && v <= 255;
}
at::Tensor new_like(const at::Tensor& t, at::IntArrayRef size, at::ScalarType type) {
    return at::empty(size, at::TensorOptions().dtype(type).device(t.device()));
}
void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }
// the caller's object where there is one, else a new one around the tensor
PyObject* give(PyObject* arg, const at::Tensor& t) {
    if (arg == Py_None) return THPVariable_Wrap(t);
    Py_INCREF(arg);
    return arg;
}

// split_weights(w, enc, w_persist or None, w_resid or None) -> (w_persist, w_resid, enc), a status that is not 0, or None
PyObject* split_weights(PyObject*, PyObject* const* args, Py_ssize_t n) {
    int32_t enc = 0;
    if (n != 4 || g_fn.split == nullptr || !small_int(args[1], enc)) Py_RETURN_NONE;
    try {
        at::Tensor w, p, r;
        if (!take(args[0], at::kHalf, 2, false, w) || !take(args[2], at::kByte, 0, true, p) || !take(args[3], at::kByte, 0, true, r))
            Py_RETURN_NONE;
        int status = 0;
        {
            WithoutGil nogil;
            if (!p.defined()) p = new_like(w, w.sizes(), at::kByte);
            if (!r.defined()) r = new_like(w, w.sizes(), at::kByte);
            status = g_fn.split(w.const_data_ptr(), p.mutable_data_ptr<uint8_t>(), r.mutable_data_ptr<uint8_t>(), w.size(0), w.size(1),
                                &enc, current_stream());
        }
        if (status != 0) return PyLong_FromLong(status);
        return Py_BuildValue("(NNi)", give(args[2], p), give(args[3], r), (int)enc);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// reconstruct(w_persist, w_resid or None, enc, out or None) -> out, a status that is not 0, or None
PyObject* reconstruct(PyObject*, PyObject* const* args, Py_ssize_t n) {
    int32_t enc = 0;
    if (n != 4 || g_fn.reconstruct == nullptr || !small_int(args[2], enc)) Py_RETURN_NONE;
    try {
        at::Tensor p, r, w;
        if (!take(args[0], at::kByte, 2, false, p) || !take(args[1], at::kByte, 0, true, r) || !take(args[3], at::kHalf, 0, true, w))
            Py_RETURN_NONE;
        int status = 0;
        {
            WithoutGil nogil;
            if (!w.defined()) w = new_like(p, p.sizes(), at::kHalf);
            status = g_fn.reconstruct(p.const_data_ptr<uint8_t>(), r.defined() ? r.const_data_ptr<uint8_t>() : nullptr, w.mutable_data_ptr(),
                                      p.size(0), p.size(1), enc, current_stream());
        }
        if (status != 0) return PyLong_FromLong(status);
        return give(args[3], w);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// moe_linear(mode, encodings, x, token_of_row or None, expert_of_row, w_persist, w_resid or None, y or None, workspace)
// -> y, a status that is not 0, or None
PyObject* moe_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr Py_ssize_t kMaxExperts = 1024;
    int32_t mode = 0, enc[kMaxExperts];
    if (n != 9 || g_fn.moe == nullptr || !small_int(args[0], mode)) Py_RETURN_NONE;
    if (!PyList_CheckExact(args[1]) && !PyTuple_CheckExact(args[1])) Py_RETURN_NONE;
    const Py_ssize_t experts = PySequence_Fast_GET_SIZE(args[1]);
    if (experts > kMaxExperts) Py_RETURN_NONE;
    for (Py_ssize_t i = 0; i < experts; ++i)
        if (!small_int(PySequence_Fast_GET_ITEM(args[1], i), enc[i])) Py_RETURN_NONE;
    try {
        at::Tensor x, token, expert, p, r, y, workspace;
        if (!take(args[2], at::kHalf, 2, false, x) || !take(args[3], at::kInt, 0, true, token) || !take(args[4], at::kInt, 0, false, expert) ||
            !take(args[5], at::kByte, 3, false, p) || !take(args[6], at::kByte, 0, true, r) || !take(args[7], at::kHalf, 0, true, y) ||
            !take(args[8], at::kByte, 0, false, workspace))
            Py_RETURN_NONE;
        if (p.size(0) != experts || x.size(1) != p.size(2)) Py_RETURN_NONE;
        const int64_t rows = expert.numel();
        int status = 0;
        {
            WithoutGil nogil;
            if (!y.defined()) y = new_like(x, {rows, p.size(1)}, at::kHalf);
            status = g_fn.moe(mode, enc, x.const_data_ptr(), token.defined() ? token.const_data_ptr<int32_t>() : nullptr,
                              expert.const_data_ptr<int32_t>(), p.const_data_ptr<uint8_t>(),
                              r.defined() ? r.const_data_ptr<uint8_t>() : nullptr, y.mutable_data_ptr(), rows, x.size(0), p.size(1),
                              p.size(2), (int32_t)experts, workspace.mutable_data_ptr(), (size_t)workspace.numel(), current_stream());
        }
        if (status != 0) return PyLong_FromLong(status);
        return give(args[7], y);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// ---- the operators of a decoder step between its linear layers ---------------------------------------------------------
// A decode step makes each of these calls for every layer, and a small one takes the GPU 2-4 us.

struct StepFunctions {
    int (*tables)(const int32_t*, const int32_t*, int64_t, const int32_t*, int64_t, int32_t*, int64_t, int64_t, int32_t, int64_t, int32_t*,
                  int32_t*, int32_t*, int64_t*, int64_t, int32_t*, void*) = nullptr;
    int (*qk)(const void*, int64_t, int64_t, int32_t, const dps_kv_cache*, const int64_t*, const int32_t*, const float*, int64_t, int32_t,
              int32_t, const void*, const void*, float, void*, int64_t, void*) = nullptr;
    int (*attention)(const void*, int64_t, int64_t, int64_t, int32_t, const dps_kv_cache*, const int32_t*, int64_t, int64_t, const int32_t*,
                     float, void*, void*, size_t, void*) = nullptr;
    int (*route)(const void*, int64_t, int32_t, int64_t, int32_t, const float*, int32_t, int32_t, int32_t, int32_t, int32_t, float, int32_t*,
                 int32_t*, float*, void*) = nullptr;
} g_step;

// set_step_functions(addresses of dps_extend_block_tables, dps_qk_norm_rope, dps_paged_attention, dps_route_experts)
PyObject* set_step_functions(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "four addresses");
        return nullptr;
    }
    void* at[4];
    for (int i = 0; i < 4; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_step.tables = reinterpret_cast<decltype(g_step.tables)>(at[0]);
    g_step.qk = reinterpret_cast<decltype(g_step.qk)>(at[1]);
    g_step.attention = reinterpret_cast<decltype(g_step.attention)>(at[2]);
    g_step.route = reinterpret_cast<decltype(g_step.route)>(at[3]);
    Py_RETURN_NONE;
}

// A tensor of the current device.
bool tensor(PyObject* arg, at::Tensor& out) {
    if (!THPVariable_CheckExact(arg)) return false;
    out = THPVariable_Unpack(arg);
    return out.is_cuda() && out.layout() == at::kStrided && out.device().index() == c10::cuda::current_device();
}
// ... contiguous, of this type and, where count >= 0, with this many elements.
bool flat(PyObject* arg, at::ScalarType type, int64_t count, bool optional, at::Tensor& out) {
    if (arg == Py_None) return optional;
    return tensor(arg, out) && out.scalar_type() == type && out.is_contiguous() && (count < 0 || out.numel() == count);
}
// ... of `dims` dimensions, the last of them dense.
bool rows(PyObject* arg, int dims, at::Tensor& out) {
    return tensor(arg, out) && out.dim() == dims && (out.size(dims - 1) <= 1 || out.stride(dims - 1) == 1);
}
bool number(PyObject* arg, double& out) {
    out = PyFloat_CheckExact(arg) ? PyFloat_AS_DOUBLE(arg) : PyLong_CheckExact(arg) ? PyLong_AsDouble(arg) : 0.0;
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return PyFloat_CheckExact(arg) || PyLong_CheckExact(arg);
}
bool whole(PyObject* arg, int64_t most, int64_t& out) {
    if (!PyLong_Check(arg)) return false;
    out = PyLong_AsLongLong(arg);
    if (out == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return out >= 0 && out <= most;
}
template <typename T>
T* data(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

bool cache_of(PyObject* k_arg, PyObject* v_arg, at::Tensor& k, at::Tensor& v, dps_kv_cache& c) {
    if (!rows(k_arg, 4, k) || !rows(v_arg, 4, v) || k.scalar_type() != v.scalar_type()) return false;
    if (k.scalar_type() != at::kHalf && k.scalar_type() != at::kBFloat16) return false;
    if (k.sizes() != v.sizes() || k.strides() != v.strides() || k.size(1) > INT32_MAX || k.size(2) > INT32_MAX || k.size(3) > INT32_MAX) return false;
    c = {k.data_ptr(), v.data_ptr(), k.size(0), k.stride(0), k.stride(1), k.stride(2), (int32_t)k.size(1), (int32_t)k.size(2), (int32_t)k.size(3),
         k.scalar_type() == at::kHalf ? DPS_TYPE_FP16 : DPS_TYPE_BF16};
    return true;
}

// extend_block_tables(lengths, new_tokens, granted or None, block_table, page_tokens, blocks, lengths_out, token_starts, positions, slots,
// granted_used) -> a status, or None
PyObject* extend_block_tables(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 11 || g_step.tables == nullptr) Py_RETURN_NONE;
    try {
        int64_t page = 0, blocks = 0;
        at::Tensor lengths, added, granted, table, after, starts, positions, slots, used;
        if (!flat(args[0], at::kInt, -1, false, lengths)) Py_RETURN_NONE;
        const int64_t b = lengths.numel();
        if (!flat(args[1], at::kInt, b, false, added) || !flat(args[2], at::kInt, -1, true, granted) || !rows(args[3], 2, table) ||
            table.scalar_type() != at::kInt || table.size(0) != b || !whole(args[4], INT32_MAX, page) || !whole(args[5], INT64_MAX, blocks) ||
            !flat(args[6], at::kInt, b, false, after) || !flat(args[7], at::kInt, b + 1, false, starts) ||
            !flat(args[8], at::kInt, -1, false, positions) || !flat(args[9], at::kLong, positions.numel(), false, slots) ||
            !flat(args[10], at::kInt, 1, false, used))
            Py_RETURN_NONE;
        int status = 0;
        {
            WithoutGil nogil;
            status = g_step.tables(data<int32_t>(lengths), data<int32_t>(added), b, data<int32_t>(granted), granted.defined() ? granted.numel() : 0,
                                   data<int32_t>(table), table.stride(0), table.size(1), (int32_t)page, blocks, data<int32_t>(after),
                                   data<int32_t>(starts), data<int32_t>(positions), data<int64_t>(slots), positions.numel(),
                                   data<int32_t>(used), current_stream());
        }
        return PyLong_FromLong(status);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// qk_norm_rope(qkv, k_cache, v_cache, slots, positions or None, cos_sin or None, q_weight or None, k_weight or None, eps, interleaved,
// q_out or None) -> q_out, a status that is not 0, or None
PyObject* qk_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 11 || g_step.qk == nullptr) Py_RETURN_NONE;
    try {
        at::Tensor qkv, k, v, slots, positions, cos_sin, qw, kw, out;
        dps_kv_cache cache;
        double eps = 0.0;
        if (!rows(args[0], 2, qkv) || !cache_of(args[1], args[2], k, v, cache) || qkv.scalar_type() != k.scalar_type()) Py_RETURN_NONE;
        const int64_t t = qkv.size(0), dim = cache.head_dim, q_width = qkv.size(1) - 2 * cache.heads * dim;
        if (dim == 0 || q_width < 0 || q_width % dim != 0 || q_width / dim > INT32_MAX) Py_RETURN_NONE;
        const int64_t heads = q_width / dim;
        if (!flat(args[3], at::kLong, t, false, slots) || !flat(args[4], at::kInt, t, true, positions) ||
            !flat(args[5], at::kFloat, -1, true, cos_sin) || (cos_sin.defined() && (cos_sin.dim() != 2 || cos_sin.size(1) > INT32_MAX)) ||
            !flat(args[6], qkv.scalar_type(), dim, true, qw) || !flat(args[7], qkv.scalar_type(), dim, true, kw) || !number(args[8], eps) ||
            !PyBool_Check(args[9]))
            Py_RETURN_NONE;
        if (args[10] != Py_None && (!rows(args[10], 3, out) || out.scalar_type() != qkv.scalar_type() || out.size(0) != t ||
                                    out.size(1) != heads || out.size(2) != dim || (heads > 1 && out.stride(1) != dim)))
            Py_RETURN_NONE;
        int status = 0;
        {
            WithoutGil nogil;
            if (!out.defined()) out = new_like(qkv, {t, heads, dim}, qkv.scalar_type());
            status = g_step.qk(qkv.data_ptr(), qkv.stride(0), t, (int32_t)heads, &cache, data<int64_t>(slots), data<int32_t>(positions),
                               data<float>(cos_sin), cos_sin.defined() ? cos_sin.size(0) : 0, cos_sin.defined() ? (int32_t)cos_sin.size(1) : 0,
                               args[9] == Py_True, data<void>(qw), data<void>(kw), (float)eps, out.data_ptr(), out.stride(0), current_stream());
        }
        if (status != 0) return PyLong_FromLong(status);
        return give(args[10], out);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// paged_attention(q, k_cache, v_cache, block_table, lengths, scale or None, out or None, workspace) -> out, a status that is not 0, or None
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 8 || g_step.attention == nullptr) Py_RETURN_NONE;
    try {
        at::Tensor q, k, v, table, lengths, out, workspace;
        dps_kv_cache cache;
        double scale = 0.0;
        if (!rows(args[0], 3, q) || !cache_of(args[1], args[2], k, v, cache) || q.scalar_type() != k.scalar_type()) Py_RETURN_NONE;
        const int64_t b = q.size(0), heads = q.size(1);
        if (q.size(2) != cache.head_dim || cache.head_dim == 0 || heads > INT32_MAX || !rows(args[3], 2, table) || table.scalar_type() != at::kInt ||
            table.size(0) != b || !flat(args[4], at::kInt, b, false, lengths) || !flat(args[6], q.scalar_type(), q.numel(), true, out) ||
            (out.defined() && out.sizes() != q.sizes()) || !flat(args[7], at::kByte, -1, false, workspace))
            Py_RETURN_NONE;
        if (args[5] == Py_None) scale = 1.0 / std::sqrt((double)cache.head_dim);
        else if (!number(args[5], scale)) Py_RETURN_NONE;
        int status = 0;
        {
            WithoutGil nogil;
            if (!out.defined()) out = new_like(q, q.sizes(), q.scalar_type());
            status = g_step.attention(q.data_ptr(), q.stride(0), q.stride(1), b, (int32_t)heads, &cache, data<int32_t>(table), table.stride(0),
                                      table.size(1), data<int32_t>(lengths), (float)scale, out.data_ptr(), workspace.data_ptr(),
                                      (size_t)workspace.numel(), current_stream());
        }
        if (status != 0) return PyLong_FromLong(status);
        return give(args[6], out);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// route_experts(logits, top_k, bias or None, scoring, groups, top_groups, renormalise, scale, token_of_row or None, expert_of_row or None,
// weights or None) -> (token_of_row, expert_of_row, weights), a status that is not 0, or None
PyObject* route_experts(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 11 || g_step.route == nullptr) Py_RETURN_NONE;
    try {
        at::Tensor logits, bias, token, expert, weights;
        int64_t top = 0, scoring = 0, groups = 0, top_groups = 0;
        double scale = 0.0;
        if (!rows(args[0], 2, logits) || !whole(args[1], 1024, top) || !whole(args[3], 255, scoring) || !whole(args[4], 1024, groups) ||
            !whole(args[5], 1024, top_groups) || !PyBool_Check(args[6]) || !number(args[7], scale))
            Py_RETURN_NONE;
        const at::ScalarType type = logits.scalar_type();
        if ((type != at::kHalf && type != at::kBFloat16 && type != at::kFloat) || logits.size(1) > INT32_MAX) Py_RETURN_NONE;
        const int64_t t = logits.size(0), count = t * top;
        if (!flat(args[2], at::kFloat, logits.size(1), true, bias) || !flat(args[8], at::kInt, count, true, token) ||
            !flat(args[9], at::kInt, count, true, expert) || !flat(args[10], at::kFloat, count, true, weights))
            Py_RETURN_NONE;
        int status = 0;
        {
            WithoutGil nogil;
            if (!token.defined()) token = new_like(logits, {count}, at::kInt);
            if (!expert.defined()) expert = new_like(logits, {count}, at::kInt);
            if (!weights.defined()) weights = new_like(logits, {t, top}, at::kFloat);
            status = g_step.route(logits.data_ptr(), logits.stride(0), type == at::kHalf ? DPS_TYPE_FP16 : type == at::kBFloat16 ? DPS_TYPE_BF16 : DPS_TYPE_FP32,
                                  t, (int32_t)logits.size(1), data<float>(bias), (int32_t)scoring, (int32_t)groups, (int32_t)top_groups,
                                  (int32_t)top, args[6] == Py_True, (float)scale, data<int32_t>(token), data<int32_t>(expert),
                                  data<float>(weights), current_stream());
        }
        if (status != 0) return PyLong_FromLong(status);
        return Py_BuildValue("(NNN)", give(args[8], token), give(args[9], expert), give(args[10], weights));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

#define DPS_FASTCALL(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    {"set_linear", set_linear, METH_O, nullptr},
    DPS_FASTCALL(set_functions),
    DPS_FASTCALL(linear),
    DPS_FASTCALL(split_weights),
    DPS_FASTCALL(reconstruct),
    DPS_FASTCALL(moe_linear),
    DPS_FASTCALL(set_step_functions),
    DPS_FASTCALL(extend_block_tables),
    DPS_FASTCALL(qk_norm_rope),
    DPS_FASTCALL(paged_attention),
    DPS_FASTCALL(route_experts),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&g_module); }
