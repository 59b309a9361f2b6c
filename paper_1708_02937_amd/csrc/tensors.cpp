// The layer of experts on torch tensors: shapes and addresses are read from the tensors, outputs and workspaces come
// from torch's allocator on the stream given, and the C entry is called.  The Python functions of experts.py choose
// device and stream and hand their arguments over in order.  A small call's time is spent on the host: one token of 4096
// columns through the norm, whose kernel takes 3.1 us, is 7.4 us a call, 11.4 with the same steps in Python (four
// tensors of torch's at about 0.9 us, the launch 2.5).
//
// Every function returns its tensors, or the status of the C call where that is not SDNN_OK.
#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <limits>

#include "sdnn.h"

namespace {

using at::ScalarType;
using at::Tensor;

constexpr ScalarType kCodes = ScalarType::Float8_e4m3fn, kScales = ScalarType::Float8_e8m0fnu;

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t pitch_of(int64_t k) { return up(k, 128) * 128; }
int64_t scale_pitch_of(int64_t k) { return up(up(k, 128), 4) * 4; }

// ---- arguments
void count(Py_ssize_t given, Py_ssize_t wanted) {
    TORCH_CHECK_TYPE(given == wanted, "expected ", wanted, " arguments, not ", given);
}

const Tensor &tensor(PyObject *o, const char *name) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a tensor");
    const Tensor &t = THPVariable_Unpack(o);
    // Results know nothing of what they were made from: a gradient would stop here without a word.
    TORCH_CHECK_VALUE(!(t.requires_grad() && c10::GradMode::is_enabled()) && !t._fw_grad(0).defined(), name,
                      " requires a gradient, and a layer of experts has none: call it under torch.no_grad(), or detach ",
                      name);
    return t;
}

int64_t integer(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

int32_t small(int64_t v, const char *name) {
    TORCH_CHECK_VALUE(v >= std::numeric_limits<int32_t>::min() && v <= std::numeric_limits<int32_t>::max(), name,
                      " is out of range: ", v);
    return (int32_t)v;
}

double real(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}

void *stream_of(PyObject *o) { return (void *)(uintptr_t)integer(o); }

ScalarType scalar_of(int64_t kind) { return kind == SDNN_TYPE_F32 ? ScalarType::Float : ScalarType::BFloat16; }

int32_t kind_of(const Tensor &t, const char *name) {
    const ScalarType s = t.scalar_type();
    TORCH_CHECK_VALUE(s == ScalarType::Float || s == ScalarType::BFloat16, name, ": float32 or bfloat16, not ", s);
    return s == ScalarType::Float ? SDNN_TYPE_F32 : SDNN_TYPE_BF16;
}

// The row stride of a matrix of that type and shape on that device, with contiguous rows.
int64_t dense(const Tensor &t, const char *name, ScalarType type, at::Device device, int64_t rows, int64_t cols) {
    TORCH_CHECK_VALUE(t.scalar_type() == type && t.device() == device && t.dim() == 2 && t.size(0) == rows &&
                          t.size(1) == cols,
                      name, " must be ", type, " of shape (", rows, ", ", cols, ") on ", device, ", not ",
                      t.scalar_type(), " of shape ", t.sizes(), " on ", t.device());
    TORCH_CHECK_VALUE(t.stride(1) == 1 || cols <= 1, name, " must have contiguous rows");
    return rows > 1 ? t.stride(0) : std::max(t.stride(0), cols);
}

// The address of a contiguous tensor of that type and shape on that device.
template <typename P>
P *packed(const Tensor &t, const char *name, ScalarType type, at::Device device, at::IntArrayRef shape) {
    TORCH_CHECK_VALUE(t.scalar_type() == type && t.device() == device && t.sizes() == shape && t.is_contiguous(), name,
                      " must be contiguous, ", type, " of shape ", shape, " on ", device, ", not ", t.scalar_type(),
                      " of shape ", t.sizes(), " on ", t.device());
    return (P *)t.data_ptr();
}

template <typename P>
P *packed(PyObject *o, const char *name, ScalarType type, at::Device device, at::IntArrayRef shape) {
    return packed<P>(tensor(o, name), name, type, device, shape);
}

Tensor empty(at::IntArrayRef shape, ScalarType type, at::Device device) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(device));
}

// ---- results
struct Unlocked {  // other Python threads run meanwhile
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

PyObject *wrapped(const Tensor &t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

template <typename... T>
PyObject *tuple_of(const T &...t) {
    PyObject *items[] = {wrapped(t)...};
    PyObject *result = PyTuple_New(sizeof...(T));
    bool fine = result != nullptr;
    for (PyObject *i : items) fine = fine && i;
    if (!fine) {
        for (PyObject *i : items) Py_XDECREF(i);
        Py_XDECREF(result);
        return nullptr;
    }
    for (size_t i = 0; i < sizeof...(T); i++) PyTuple_SET_ITEM(result, i, items[i]);
    return result;
}

// ---- calls
// x, block_rows, stream -> codes, scales
PyObject *quantize_blocks(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 3);
    const Tensor &x = tensor(args[0], "x");
    const int32_t block_rows = small(integer(args[1]), "block_rows");
    void *const stream = stream_of(args[2]);
    TORCH_CHECK_VALUE(x.dim() >= 2 && x.is_contiguous(), "x must be contiguous, (..., rows, k)");
    const int32_t kind = kind_of(x, "x");
    const int64_t rows = x.size(-2), k = x.size(-1);
    const int64_t each = rows * k;
    std::vector<int64_t> shape = x.sizes().vec();
    shape.back() = pitch_of(k);
    const Tensor codes = empty(shape, kCodes, x.device());
    shape[shape.size() - 2] = block_rows == 1 ? rows : up(rows, 128);
    shape.back() = scale_pitch_of(k);
    const Tensor scales = empty(shape, kScales, x.device());
    sdnn_status s;
    {
        Unlocked u;
        s = sdnn_quantize_blocks(each ? x.numel() / each : 0, rows, k, block_rows, kind, x.data_ptr(), k,
                                 (uint8_t *)codes.data_ptr(), (uint8_t *)scales.data_ptr(), stream);
    }
    return s ? PyLong_FromLong(s) : tuple_of(codes, scales);
    END_HANDLE_TH_ERRORS
}

// x, gamma, eps, residual, normed, out_sum, stream -> codes, scales, sum, normed
PyObject *norm_quantize(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 7);
    const Tensor &x = tensor(args[0], "x");
    const float eps = (float)real(args[2]);
    const bool normed = PyObject_IsTrue(args[4]) == 1;
    void *const stream = stream_of(args[6]);
    TORCH_CHECK_VALUE(x.dim() == 2, "x must be a matrix");
    const int64_t rows = x.size(0), k = x.size(1);
    const at::Device device = x.device();
    const ScalarType type = x.scalar_type();
    const int32_t kind = kind_of(x, "x");
    const int64_t ldx = dense(x, "x", type, device, rows, k);
    const float *gamma = packed<float>(args[1], "gamma", ScalarType::Float, device, {k});
    const void *residual = nullptr;
    int64_t ldr = 0, lds = 0;
    Tensor sum, z;
    if (args[3] != Py_None) {
        const Tensor &r = tensor(args[3], "residual");
        ldr = dense(r, "residual", type, device, rows, k);
        residual = r.data_ptr();
        if (args[5] == Py_None) {
            sum = empty({rows, k}, type, device), lds = k;
        } else {
            sum = tensor(args[5], "out_sum");
            lds = dense(sum, "out_sum", type, device, rows, k);
        }
    } else {
        TORCH_CHECK_VALUE(args[5] == Py_None, "out_sum without a residual");
    }
    if (normed) z = empty({rows, k}, type, device);
    const Tensor codes = empty({rows, pitch_of(k)}, kCodes, device);
    const Tensor scales = empty({rows, scale_pitch_of(k)}, kScales, device);
    sdnn_status s;
    {
        Unlocked u;
        s = sdnn_norm_quantize(rows, k, kind, x.data_ptr(), ldx, residual, ldr, gamma, eps,
                               sum.defined() ? sum.data_ptr() : nullptr, lds, normed ? z.data_ptr() : nullptr, k,
                               (uint8_t *)codes.data_ptr(), (uint8_t *)scales.data_ptr(), stream);
    }
    return s ? PyLong_FromLong(s) : tuple_of(codes, scales, sum, z);
    END_HANDLE_TH_ERRORS
}

// a, a_scale, w, w_scale, k, bias, ymax, kind, out, stream -> y
PyObject *product_blocks(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 10);
    const Tensor &a = tensor(args[0], "a"), &w = tensor(args[2], "w");
    const int64_t k = integer(args[4]), kind = integer(args[7]);
    const bool clamp = args[6] != Py_None;
    const float ymax = clamp ? (float)real(args[6]) : 0.0f;
    void *const stream = stream_of(args[9]);
    TORCH_CHECK_VALUE(a.dim() == 2 && w.dim() == 2, "a and w must be matrices");
    const int64_t rows = a.size(0), cols = w.size(0), pitch = pitch_of(k), spitch = scale_pitch_of(k);
    const at::Device device = a.device();
    const ScalarType type = scalar_of(kind);
    const uint8_t *pa = packed<uint8_t>(a, "a", kCodes, device, {rows, pitch});
    const uint8_t *psa = packed<uint8_t>(args[1], "a_scale", kScales, device, {rows, spitch});
    const uint8_t *pw = packed<uint8_t>(w, "w", kCodes, device, {cols, pitch});
    const uint8_t *psw = packed<uint8_t>(args[3], "w_scale", kScales, device, {up(cols, 128), spitch});
    const float *bias =
        args[5] == Py_None ? nullptr : packed<float>(args[5], "bias", ScalarType::Float, device, {cols});
    const Tensor y = args[8] == Py_None ? empty({rows, cols}, type, device) : tensor(args[8], "out");
    const int64_t ldy = args[8] == Py_None ? cols : dense(y, "out", type, device, rows, cols);
    sdnn_status s;
    {
        Unlocked u;
        s = sdnn_product_blocks(rows, cols, k, pa, psa, pw, psw, bias, clamp, ymax, (int32_t)kind, y.data_ptr(), ldy,
                                stream);
    }
    return s ? PyLong_FromLong(s) : wrapped(y);
    END_HANDLE_TH_ERRORS
}

// logits, k, score, bias, groups, groups_kept, group_best, normalize, factor, stream -> ids, weight, offsets, order
PyObject *route(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 10);
    const Tensor &logits = tensor(args[0], "logits");
    const int32_t chosen = small(integer(args[1]), "k"), score = (int32_t)integer(args[2]);
    const int32_t groups = small(integer(args[4]), "groups"), kept = small(integer(args[5]), "groups_kept"),
                  best = small(integer(args[6]), "group_best");
    const int32_t normalize = PyObject_IsTrue(args[7]) == 1;
    const float factor = (float)real(args[8]);
    void *const stream = stream_of(args[9]);
    TORCH_CHECK_VALUE(logits.dim() == 2, "logits must be tokens x experts");
    TORCH_CHECK_VALUE(chosen >= 1, "k must be at least 1");
    const int64_t tokens = logits.size(0);
    const int32_t experts = small(logits.size(1), "experts"), kind = kind_of(logits, "logits");
    const at::Device device = logits.device();
    const int64_t ldl = dense(logits, "logits", logits.scalar_type(), device, tokens, experts);
    const float *bias =
        args[3] == Py_None ? nullptr : packed<float>(args[3], "bias", ScalarType::Float, device, {experts});
    int64_t need = 0;
    sdnn_status s = sdnn_route_workspace_size(tokens, experts, chosen, &need);
    if (s) return PyLong_FromLong(s);
    const Tensor ids = empty({tokens, chosen}, ScalarType::Int, device);
    const Tensor weight = empty({tokens, chosen}, ScalarType::Float, device);
    const Tensor offsets = empty({experts + 1}, ScalarType::Int, device);
    const Tensor order = empty({tokens * chosen}, ScalarType::Int, device);
    Tensor ws;
    if (need) ws = empty({need}, ScalarType::Byte, device);
    {
        Unlocked u;
        s = sdnn_route(tokens, experts, chosen, score, kind, logits.data_ptr(), ldl, bias, groups, kept, best,
                       normalize, factor, (int32_t *)ids.data_ptr(), (float *)weight.data_ptr(),
                       (int32_t *)offsets.data_ptr(), (int32_t *)order.data_ptr(), need ? ws.data_ptr() : nullptr,
                       need, stream);
    }
    return s ? PyLong_FromLong(s) : tuple_of(ids, weight, offsets, order);
    END_HANDLE_TH_ERRORS
}

// a, a_scale, ids, weight, offsets, order, w_in, w_in_scale, w_out, w_out_scale, width, inner, residual, kind, out, ws,
// stream -> out
PyObject *experts_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 17);
    const Tensor &a = tensor(args[0], "a"), &ids = tensor(args[2], "ids"), &w_in = tensor(args[6], "w_in");
    const int64_t width = integer(args[10]), inner = integer(args[11]), kind = integer(args[13]);
    void *const stream = stream_of(args[16]);
    TORCH_CHECK_VALUE(a.dim() == 2, "a must be a matrix");
    TORCH_CHECK_VALUE(ids.dim() == 2, "ids must be tokens x chosen");
    TORCH_CHECK_VALUE(w_in.dim() == 4, "w_in must be (experts, 2, inner, pitch of width)");
    const at::Device device = a.device();
    const ScalarType type = scalar_of(kind);
    const int64_t tokens = a.size(0);
    const int32_t experts = small(w_in.size(0), "experts"), chosen = small(ids.size(1), "chosen");
    const int64_t pitch = pitch_of(width), spitch = scale_pitch_of(width);
    const int64_t pitch_f = pitch_of(inner), spitch_f = scale_pitch_of(inner);
    const uint8_t *pa = packed<uint8_t>(a, "a", kCodes, device, {tokens, pitch});
    const uint8_t *psa = packed<uint8_t>(args[1], "a_scale", kScales, device, {tokens, spitch});
    const int32_t *pi = packed<int32_t>(ids, "ids", ScalarType::Int, device, {tokens, chosen});
    const float *pw = packed<float>(args[3], "weight", ScalarType::Float, device, {tokens, chosen});
    const int32_t *pf = packed<int32_t>(args[4], "offsets", ScalarType::Int, device, {experts + 1});
    const int32_t *po = packed<int32_t>(args[5], "order", ScalarType::Int, device, {tokens * chosen});
    const uint8_t *p1 = packed<uint8_t>(w_in, "w_in", kCodes, device, {experts, 2, inner, pitch});
    const uint8_t *ps1 = packed<uint8_t>(args[7], "w_in_scale", kScales, device, {experts, 2, up(inner, 128), spitch});
    const uint8_t *p2 = packed<uint8_t>(args[8], "w_out", kCodes, device, {experts, width, pitch_f});
    const uint8_t *ps2 = packed<uint8_t>(args[9], "w_out_scale", kScales, device, {experts, up(width, 128), spitch_f});
    const void *residual = nullptr;
    int64_t ldr = 0;
    if (args[12] != Py_None) {
        const Tensor &r = tensor(args[12], "residual");
        ldr = dense(r, "residual", type, device, tokens, width);
        residual = r.data_ptr();
    }
    const Tensor out = args[14] == Py_None ? empty({tokens, width}, type, device) : tensor(args[14], "out");
    const int64_t ldo = args[14] == Py_None ? width : dense(out, "out", type, device, tokens, width);
    Tensor ws;
    sdnn_status s;
    if (args[15] == Py_None) {
        int64_t need = 0;
        s = sdnn_experts_workspace_size(tokens, width, inner, experts, chosen, (int32_t)kind, &need);
        if (s) return PyLong_FromLong(s);
        ws = empty({need}, ScalarType::Byte, device);
    } else {
        ws = tensor(args[15], "ws");
        TORCH_CHECK_VALUE(ws.device() == device && ws.scalar_type() == ScalarType::Byte && ws.is_contiguous(),
                          "ws must be a contiguous uint8 tensor on the same device");
    }
    {
        Unlocked u;
        s = sdnn_experts_forward(tokens, width, inner, experts, chosen, pa, psa, pi, pw, pf, po, p1, ps1, p2, ps2,
                                 (int32_t)kind, residual, ldr, out.data_ptr(), ldo, ws.data_ptr(), ws.numel(), stream);
    }
    return s ? PyLong_FromLong(s) : wrapped(out);
    END_HANDLE_TH_ERRORS
}

#define SDNN_CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SDNN_CALL(quantize_blocks), SDNN_CALL(norm_quantize),   SDNN_CALL(product_blocks),
                         SDNN_CALL(route),           SDNN_CALL(experts_forward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
