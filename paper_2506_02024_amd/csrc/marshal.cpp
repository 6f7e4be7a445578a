// Marshalling of the calls that stand between a layer's linears (norm, cache write, attention), of linears with an epilogue and of mixtures of experts: torch tensors to the arguments of
// the C ABI, with the checks of the Python binding.  No arithmetic.  In Python these checks cost more than a small kernel takes: 5
// to 6 us of host time per call of 15 to 21 arguments, of them 1.2 in ctypes; here about 0.5.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/nestedfp.h"

#include <algorithm>

namespace {

decltype(&nestedfp_add_rms_norm) add_rms_norm_fn;
decltype(&nestedfp_rope_append) rope_append_fn;
decltype(&nestedfp_paged_attention) paged_attention_fn;
decltype(&nestedfp_linear_fused) linear_fused_fn;
decltype(&nestedfp_linear_fused_prequantized) linear_fused_prequantized_fn;
decltype(&nestedfp_moe_route) moe_route_fn;
decltype(&nestedfp_moe) moe_fn;

// A wrong argument: its Python error is set.
struct Refused {};
[[noreturn]] void refuse(const char *name, const char *what) {
    PyErr_Format(PyExc_ValueError, "%s must be %s", name, what);
    throw Refused{};
}

const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) refuse(name, "a tensor");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) refuse(name, "on the GPU");
    return t;
}

struct Rows {
    int64_t rows = 0, cols = 0, ld = 0;
    void *at = nullptr;
    bool dense() const { return rows < 2 || ld == cols; }      // (one row is, whatever its stride, as for torch)
};
Rows rows_of(PyObject *o, const char *name, at::ScalarType type, const char *what) {
    const at::Tensor &t = tensor(o, name);
    if (t.dim() != 2 || t.scalar_type() != type || (t.stride(1) != 1 && t.size(1) > 1)) refuse(name, what);
    Rows r;
    r.rows = t.size(0);
    r.cols = t.size(1);
    r.ld = r.rows > 1 ? t.stride(0) : std::max(t.stride(0), r.cols);
    r.at = t.data_ptr();
    return r;
}
// one that may be missing, of a given shape
Rows like(PyObject *o, const char *name, const Rows &shape) {
    if (o == Py_None) return Rows();
    const Rows r = rows_of(o, name, at::kHalf, "float16 [M,K] with unit inner stride");
    if (r.rows != shape.rows || r.cols != shape.cols) refuse(name, "of the shape of the input");
    return r;
}
void *dense(PyObject *o, const char *name, at::ScalarType type, int64_t count, const char *what) {
    const at::Tensor &t = tensor(o, name);
    if (t.scalar_type() != type || t.numel() != count || !t.is_contiguous()) refuse(name, what);
    return t.data_ptr();
}
int64_t whole(PyObject *o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
}
float real(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return (float)v;
}
void *address(PyObject *o) { return reinterpret_cast<void *>(whole(o)); }

// the description of a cache, by its address in the binding's object; 0 stands for storage that is not on the GPU
const nestedfp_kv_cache *cache_of(PyObject *o) {
    const auto *cache = static_cast<const nestedfp_kv_cache *>(address(o));
    if (cache == nullptr) refuse("cache", "on the GPU");
    return cache;
}

Rows heads_of(PyObject *o, const char *name, int dim) {
    const Rows r = rows_of(o, name, at::kHalf, "float16 [tokens, heads * head_dim]");
    if (r.cols == 0 || r.cols % dim != 0) refuse(name, "float16 [tokens, heads * head_dim]");
    return r;
}

template <typename F>
PyObject *call(Py_ssize_t given, Py_ssize_t wanted, F &&f) {
    if (given != wanted) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Refused &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    }
}

// X, weight, eps, residual, sum_out, out, Xq, scales, stream
PyObject *add_rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return call(n, 9, [&] {
        const Rows x = rows_of(a[0], "X", at::kHalf, "float16 [M,K] with unit inner stride");
        const void *w = dense(a[1], "weight", at::kHalf, x.cols, "a contiguous float16 [K] tensor");
        const Rows r = like(a[3], "residual", x), s = like(a[4], "sum_out", x), y = like(a[5], "out", x);
        void *q = nullptr, *scales = nullptr;
        if (a[6] != Py_None) {
            const Rows codes = rows_of(a[6], "Xq", at::kByte, "a contiguous uint8 [M,K] tensor");
            if (codes.rows != x.rows || codes.cols != x.cols || !codes.dense()) refuse("Xq", "a contiguous uint8 [M,K] tensor");
            q = codes.at;
            scales = dense(a[7], "scales", at::kFloat, x.rows, "a contiguous float32 [M] tensor");
        }
        return add_rms_norm_fn((const uint16_t *)x.at, x.rows, x.cols, x.ld, (const uint16_t *)r.at, r.ld, (const uint16_t *)w, real(a[2]),
                               (uint16_t *)s.at, s.ld, (uint16_t *)y.at, y.ld, (uint8_t *)q, (float *)scales, address(a[8]));
    });
}

// q, k, v, positions, slots, description of the cache, cos, sin, out, stream
PyObject *rope_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return call(n, 10, [&] {
        const auto *cache = cache_of(a[5]);
        const int dim = cache->head_dim;
        const Rows q = heads_of(a[0], "q", dim), k = heads_of(a[1], "k", dim), v = heads_of(a[2], "v", dim);
        if (k.rows != q.rows || v.rows != q.rows || k.cols != (int64_t)cache->kv_heads * dim || v.cols != k.cols)
            refuse("k and v", "[tokens, kv_heads * head_dim] of the cache");
        const void *positions = nullptr, *slots = dense(a[4], "slots", at::kInt, q.rows, "a contiguous int32 tensor, one for every token");
        Rows cos, sin;
        if ((a[6] == Py_None) != (a[7] == Py_None)) refuse("cos and sin", "given together");
        if (a[6] != Py_None) {
            const char *what = "a contiguous float32 [positions, rotary_dim / 2] tensor";
            cos = rows_of(a[6], "cos", at::kFloat, what);
            sin = rows_of(a[7], "sin", at::kFloat, what);
            if (!cos.dense() || !sin.dense()) refuse("cos and sin", "contiguous");
            if (sin.rows != cos.rows || sin.cols != cos.cols) refuse("sin", "of the shape of cos");
            positions = dense(a[3], "positions", at::kInt, q.rows, "a contiguous int32 tensor, one for every token");
        }
        const Rows out = heads_of(a[8], "out", dim);
        if (out.rows != q.rows || out.cols != q.cols) refuse("out", "of the shape of q");
        return rope_append_fn((const uint16_t *)q.at, q.ld, (const uint16_t *)k.at, k.ld, (const uint16_t *)v.at, v.ld, q.rows, q.cols / dim,
                              (const float *)cos.at, (const float *)sin.at, cos.rows, 2 * cos.cols, (const int32_t *)positions,
                              (const int32_t *)slots, (uint16_t *)out.at, out.ld, cache, address(a[9]));
    });
}

// q, description of the cache, table, lens, starts, max_new, max_len, scale, window, sinks, out, workspace, stream
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return call(n, 13, [&] {
        const auto *cache = cache_of(a[1]);
        const int dim = cache->head_dim;
        const Rows q = heads_of(a[0], "q", dim), out = heads_of(a[10], "out", dim);
        if (out.rows != q.rows || out.cols != q.cols) refuse("out", "of the shape of q");
        Rows table = rows_of(a[2], "table", at::kInt, "int32 [batch, columns] with unit inner stride");
        if (table.rows <= 1 || table.cols == 0) table.ld = std::max(table.ld, table.cols);
        const void *lens = dense(a[3], "lens", at::kInt, table.rows, "a contiguous int32 tensor, one for every row of the table");
        const void *starts = a[4] == Py_None ? nullptr : dense(a[4], "starts", at::kInt, table.rows + 1, "a contiguous int32 [batch + 1] tensor");
        const at::Tensor &workspace = tensor(a[11], "workspace");
        return paged_attention_fn((const uint16_t *)q.at, q.rows, q.ld, q.cols / dim, cache, (const int32_t *)table.at, table.ld, table.cols,
                                  (const int32_t *)lens, table.rows, (const int32_t *)starts, whole(a[5]), whole(a[6]), real(a[7]), whole(a[8]),
                                  whole(a[9]), (uint16_t *)out.at, out.ld, workspace.data_ptr(), workspace.nbytes(), address(a[12]));
    });
}

// X or codes, scales, description of the layer, mode, act_scale, bias, activation, gated, residual, out, workspace, stream
PyObject *linear_fused(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return call(n, 12, [&] {
        const auto *layer = static_cast<const nestedfp_layer *>(address(a[2]));
        nestedfp_epilogue e = nestedfp_epilogue();
        e.activation = (int32_t)whole(a[6]);
        e.gated = PyObject_IsTrue(a[7]) == 1;
        const bool codes = a[1] != Py_None;
        if (codes && whole(a[3]) != NESTEDFP_MODE_FP8) refuse("mode", "FP8 mode where X is codes");
        if (codes && a[4] != Py_None) refuse("act_scale", "None where X is codes, which have scales");
        const char *what = codes ? "contiguous uint8 [M,K] codes, K as the layer's" : "float16 [M,K] with unit inner stride, K as the layer's";
        const Rows x = rows_of(a[0], "X", codes ? at::kByte : at::kHalf, what);
        if (x.cols != layer->K || (codes && !x.dense())) refuse("X", what);
        if (e.gated && layer->N % 2 != 0) refuse("a gated layer's rows", "gate and up rows in turn");
        Rows shape;
        shape.rows = x.rows;
        shape.cols = e.gated ? layer->N / 2 : layer->N;
        const Rows residual = like(a[8], "residual", shape), out = like(a[9], "out", shape);
        if (out.at == nullptr && shape.rows * shape.cols > 0) refuse("out", "float16 [M, outputs]");
        e.bias = a[5] == Py_None ? nullptr : (const uint16_t *)dense(a[5], "bias", at::kHalf, layer->N, "a contiguous float16 [N] tensor");
        e.residual = (const uint16_t *)residual.at;
        e.ldr = residual.ld;
        const at::Tensor &workspace = tensor(a[10], "workspace");
        if (codes)
            return linear_fused_prequantized_fn((const uint8_t *)x.at, (const float *)dense(a[1], "scales", at::kFloat, x.rows, "a contiguous float32 [M] tensor"),
                                                x.rows, layer, &e, (uint16_t *)out.at, out.ld, workspace.data_ptr(), workspace.nbytes(), address(a[11]));
        const float *scale = a[4] == Py_None ? nullptr : (const float *)dense(a[4], "act_scale", at::kFloat, 1, "a float32 tensor of one value");
        return linear_fused_fn((const uint16_t *)x.at, x.rows, x.ld, layer, (int)whole(a[3]), scale, &e, (uint16_t *)out.at, out.ld,
                               workspace.data_ptr(), workspace.nbytes(), address(a[11]));
    });
}

// X, router, top_k, scoring, renormalize, factor, bias, ids, weights, workspace, stream
PyObject *moe_route(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return call(n, 11, [&] {
        const Rows x = rows_of(a[0], "X", at::kHalf, "float16 [M,K] with unit inner stride");
        const Rows r = rows_of(a[1], "router", at::kHalf, "float16 [experts,K] with unit inner stride");
        if (r.cols != x.cols) refuse("router", "float16 [experts,K], K as that of X");
        const int64_t top_k = whole(a[2]);
        const char *what = "a contiguous [M,top_k] tensor, ids int32 and weights float32";
        const Rows shape = rows_of(a[7], "ids", at::kInt, what), shape_w = rows_of(a[8], "weights", at::kFloat, what);
        if (shape.rows != x.rows || shape.cols != top_k || shape_w.rows != x.rows || shape_w.cols != top_k) refuse("ids and weights", what);
        void *ids = dense(a[7], "ids", at::kInt, x.rows * top_k, what), *weights = dense(a[8], "weights", at::kFloat, x.rows * top_k, what);
        const void *bias = a[6] == Py_None ? nullptr : dense(a[6], "bias", at::kFloat, r.rows, "a contiguous float32 [experts] tensor");
        const at::Tensor &workspace = tensor(a[9], "workspace");
        return moe_route_fn((const uint16_t *)x.at, x.rows, x.cols, x.ld, (const uint16_t *)r.at, r.rows, r.ld, top_k, (int)whole(a[3]),
                            PyObject_IsTrue(a[4]) == 1, real(a[5]), (const float *)bias, (int32_t *)ids, (float *)weights, workspace.data_ptr(),
                            workspace.nbytes(), address(a[10]));
    });
}

// X, description of the experts, mode, ids, weights, residual, out, workspace, stream
PyObject *moe(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return call(n, 9, [&] {
        const auto *experts = static_cast<const nestedfp_experts *>(address(a[1]));
        const Rows x = rows_of(a[0], "X", at::kHalf, "float16 [M, hidden] with unit inner stride");
        if (x.cols != experts->hidden) refuse("X", "float16 [M, hidden] of the experts");
        const char *what = "contiguous [M,top_k] tensors, ids int32 and weights float32";
        const Rows ids = rows_of(a[3], "ids", at::kInt, what), weights = rows_of(a[4], "weights", at::kFloat, what);
        if (ids.rows != x.rows || weights.rows != x.rows || ids.cols != weights.cols || !ids.dense() || !weights.dense())
            refuse("ids and weights", what);
        const Rows residual = like(a[5], "residual", x), out = like(a[6], "out", x);
        const at::Tensor &workspace = tensor(a[7], "workspace");
        return moe_fn((const uint16_t *)x.at, x.rows, x.ld, experts, (int)whole(a[2]), (const int32_t *)ids.at, (const float *)weights.at, ids.cols,
                      (const uint16_t *)residual.at, residual.ld, (uint16_t *)out.at, out.ld, workspace.data_ptr(), workspace.nbytes(), address(a[8]));
    });
}

// addresses of the entry points in the library that the binding has loaded
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return call(n, 7, [&] {
        add_rms_norm_fn = reinterpret_cast<decltype(add_rms_norm_fn)>(address(a[0]));
        rope_append_fn = reinterpret_cast<decltype(rope_append_fn)>(address(a[1]));
        paged_attention_fn = reinterpret_cast<decltype(paged_attention_fn)>(address(a[2]));
        linear_fused_fn = reinterpret_cast<decltype(linear_fused_fn)>(address(a[3]));
        linear_fused_prequantized_fn = reinterpret_cast<decltype(linear_fused_prequantized_fn)>(address(a[4]));
        moe_route_fn = reinterpret_cast<decltype(moe_route_fn)>(address(a[5]));
        moe_fn = reinterpret_cast<decltype(moe_fn)>(address(a[6]));
        return 0;
    });
}

PyCFunction fast(PyObject *(*f)(PyObject *, PyObject *const *, Py_ssize_t)) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)); }
PyMethodDef methods[] = {{"bind", fast(bind), METH_FASTCALL, nullptr},
                         {"add_rms_norm", fast(add_rms_norm), METH_FASTCALL, nullptr},
                         {"rope_append", fast(rope_append), METH_FASTCALL, nullptr},
                         {"paged_attention", fast(paged_attention), METH_FASTCALL, nullptr},
                         {"linear_fused", fast(linear_fused), METH_FASTCALL, nullptr},
                         {"moe_route", fast(moe_route), METH_FASTCALL, nullptr},
                         {"moe", fast(moe), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
