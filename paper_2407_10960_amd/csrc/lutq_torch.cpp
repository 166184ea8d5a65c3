// Plain calls of the Python binding in native code: argument checks, raw pointers, current stream, call.
//
// In Python these cost about twice what the smallest launches take on the GPU (8B O projection, M = 1: 9.9 us a call
// among others for a kernel of 4.4 us; through this module 4.3 us).  A call that is not plain -- an argument that is no ordinary
// CUDA tensor, or that any check of the binding would refuse -- is answered with -1 before anything is done, and the
// binding's own code takes it from there (and says what is wrong with it).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/DispatchKeySet.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "lutq.h"

namespace {

decltype(&lutq_packed_bytes) packed_bytes = nullptr;
decltype(&lutq_matmul) matmul = nullptr;
decltype(&lutq_matmul_static) matmul_static = nullptr;
decltype(&lutq_matmul_channel) matmul_channel = nullptr;
decltype(&lutq_matmul_pairs) matmul_pairs = nullptr;
decltype(&lutq_matmul_quads) matmul_quads = nullptr;
decltype(&lutq_quantize) quantize = nullptr;
decltype(&lutq_dequant) dequant = nullptr;
decltype(&lutq_mx4_packed_bytes) mx4_packed_bytes = nullptr;
decltype(&lutq_mx4_quantize) mx4_quantize = nullptr;
decltype(&lutq_mx4_quantize_packed) mx4_quantize_packed = nullptr;
decltype(&lutq_mx4_dequant) mx4_dequant = nullptr;
decltype(&lutq_mx4_dequant_packed) mx4_dequant_packed = nullptr;
decltype(&lutq_mx4_matmul) mx4_matmul = nullptr;
decltype(&lutq_mx4_matmul_grouped) mx4_matmul_grouped = nullptr;
decltype(&lutq_fp8_quantize) fp8_quantize = nullptr;
decltype(&lutq_fp8_quantize_weights) fp8_quantize_weights = nullptr;
decltype(&lutq_fp8_quantize_columns) fp8_quantize_columns = nullptr;
decltype(&lutq_fp8_dequant) fp8_dequant = nullptr;
decltype(&lutq_fp8_dequant_weights) fp8_dequant_weights = nullptr;
decltype(&lutq_fp8_matmul) fp8_matmul = nullptr;
decltype(&lutq_fp8_matmul_grouped) fp8_matmul_grouped = nullptr;
decltype(&lutq_fp8_gated) fp8_gated = nullptr;
decltype(&lutq_fp8_gated_grouped) fp8_gated_grouped = nullptr;
decltype(&lutq_fp8_gated_grad) fp8_gated_grad = nullptr;
decltype(&lutq_fp8_weight_grad) fp8_weight_grad = nullptr;

// the functions of liblutq.so by address, in the order of the declarations above
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr Py_ssize_t kCount = 26;
    void* p[kCount];
    if (n != kCount) { PyErr_SetString(PyExc_TypeError, "twenty-six addresses"); return nullptr; }
    for (int i = 0; i < kCount; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address"); return nullptr; }
    }
    packed_bytes = reinterpret_cast<decltype(packed_bytes)>(p[0]);
    matmul = reinterpret_cast<decltype(matmul)>(p[1]);
    matmul_static = reinterpret_cast<decltype(matmul_static)>(p[2]);
    matmul_channel = reinterpret_cast<decltype(matmul_channel)>(p[3]);
    matmul_pairs = reinterpret_cast<decltype(matmul_pairs)>(p[4]);
    matmul_quads = reinterpret_cast<decltype(matmul_quads)>(p[5]);
    quantize = reinterpret_cast<decltype(quantize)>(p[6]);
    dequant = reinterpret_cast<decltype(dequant)>(p[7]);
    mx4_packed_bytes = reinterpret_cast<decltype(mx4_packed_bytes)>(p[8]);
    mx4_quantize = reinterpret_cast<decltype(mx4_quantize)>(p[9]);
    mx4_quantize_packed = reinterpret_cast<decltype(mx4_quantize_packed)>(p[10]);
    mx4_dequant = reinterpret_cast<decltype(mx4_dequant)>(p[11]);
    mx4_dequant_packed = reinterpret_cast<decltype(mx4_dequant_packed)>(p[12]);
    mx4_matmul = reinterpret_cast<decltype(mx4_matmul)>(p[13]);
    mx4_matmul_grouped = reinterpret_cast<decltype(mx4_matmul_grouped)>(p[14]);
    fp8_quantize = reinterpret_cast<decltype(fp8_quantize)>(p[15]);
    fp8_quantize_weights = reinterpret_cast<decltype(fp8_quantize_weights)>(p[16]);
    fp8_quantize_columns = reinterpret_cast<decltype(fp8_quantize_columns)>(p[17]);
    fp8_dequant = reinterpret_cast<decltype(fp8_dequant)>(p[18]);
    fp8_dequant_weights = reinterpret_cast<decltype(fp8_dequant_weights)>(p[19]);
    fp8_matmul = reinterpret_cast<decltype(fp8_matmul)>(p[20]);
    fp8_matmul_grouped = reinterpret_cast<decltype(fp8_matmul_grouped)>(p[21]);
    fp8_gated = reinterpret_cast<decltype(fp8_gated)>(p[22]);
    fp8_gated_grouped = reinterpret_cast<decltype(fp8_gated_grouped)>(p[23]);
    fp8_gated_grad = reinterpret_cast<decltype(fp8_gated_grad)>(p[24]);
    fp8_weight_grad = reinterpret_cast<decltype(fp8_weight_grad)>(p[25]);
    Py_RETURN_NONE;
}

// an ordinary dense CUDA tensor (no subclass, no functorch or functionalisation wrapper) that is contiguous, or null
const at::Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    static const c10::DispatchKeySet wrappers({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                               c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize});
    if (!t.defined() || t.layout() != c10::kStrided || t.unsafeGetTensorImpl()->key_set().has_any(wrappers)) return nullptr;
    return t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

int dtype_code(const at::Tensor& t) {
    return t.scalar_type() == at::kHalf ? LUTQ_F16 : t.scalar_type() == at::kBFloat16 ? LUTQ_BF16 : -1;
}

bool small_int(PyObject* o, long lo, long hi, int* out) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over || v < lo || v > hi) return false;
    *out = (int)v;
    return true;
}

bool shape_is(const at::Tensor& t, int64_t a, int64_t b) { return t.dim() == 2 && t.size(0) == a && t.size(1) == b; }

void* current_stream() { return static_cast<void*>(c10::hip::getCurrentHIPStream().stream()); }

// A torch call that throws (a nested tensor asked for an irregular size, storage that may not be read, no device) makes the call one
// that is not plain: no exception leaves through the C entry, and the binding's own code meets the same refusal and raises it.
template <typename F> PyObject* answer(F f) {
    try { return f(); } catch (...) { return PyLong_FromLong(-1); }
}

struct WithoutGil {
    PyThreadState* state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

enum Kind { kMatmul = 0, kStatic = 1, kChannel = 2, kPairs = 3, kQuads = 4 };

// (kind, X, packed, scales, lut, bits, group_size, Y, workspace or None) -> status, or -1
PyObject* mm(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    int kind, bits, group;
    if (!matmul || n != 9 || !small_int(args[0], 0, 4, &kind) || !small_int(args[5], 2, 4, &bits) || !small_int(args[6], 1, 1 << 16, &group))
        return PyLong_FromLong(-1);
    const at::Tensor *X = plain(args[1]), *packed = plain(args[2]), *scales = plain(args[3]), *lut = plain(args[4]),
                     *Y = plain(args[7]), *ws = kind == kStatic ? nullptr : plain(args[8]);
    if (!X || !packed || !scales || !lut || !Y || (kind != kStatic && !ws)) return PyLong_FromLong(-1);
    const int code = dtype_code(*X);
    if (code < 0 || dtype_code(*scales) != code || dtype_code(*lut) != code || dtype_code(*Y) != code || X->dim() != 2 || scales->dim() != 2)
        return PyLong_FromLong(-1);
    const int64_t M = X->size(0), K = X->size(1), N = scales->size(0);
    const bool table = kind == kChannel ? shape_is(*lut, N, 1 << bits)
                     : kind == kPairs   ? bits == 4 && shape_is(*lut, 256, 2)
                     : kind == kQuads   ? bits == 2 && shape_is(*lut, 256, 4)
                                        : lut->numel() == (1 << bits);
    if (!table || scales->size(1) * group != K || !shape_is(*Y, M, N) || packed->numel() != (int64_t)packed_bytes(N, K, bits, group))
        return PyLong_FromLong(-1);
    const void *x = X->data_ptr(), *p = packed->data_ptr(), *s = scales->data_ptr(), *l = lut->data_ptr();
    void *y = Y->data_ptr(), *w = ws ? ws->data_ptr() : nullptr, *stream = current_stream();
    const size_t wb = ws ? (size_t)ws->numel() * ws->element_size() : 0;
    const lutq_dtype dt = (lutq_dtype)code;
    lutq_status st = LUTQ_OK;
    {
        WithoutGil released;
        switch (kind) {
            case kMatmul: st = matmul(x, p, s, l, bits, group, M, N, K, dt, y, w, wb, stream); break;
            case kStatic: st = matmul_static(x, p, s, l, bits, group, M, N, K, dt, y, stream, nullptr); break;
            case kChannel: st = matmul_channel(x, p, s, l, bits, group, M, N, K, dt, y, w, wb, stream); break;
            case kPairs: st = matmul_pairs(x, p, s, l, group, M, N, K, dt, y, w, wb, stream); break;
            case kQuads: st = matmul_quads(x, p, s, l, group, M, N, K, dt, y, w, wb, stream); break;
        }
    }
    return PyLong_FromLong((long)st);
}); }

// (W, lut, bits, group_size, scales_out, packed_out) -> status, or -1
PyObject* quant(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    int bits, group;
    if (!quantize || n != 6 || !small_int(args[2], 2, 4, &bits) || !small_int(args[3], 1, 1 << 16, &group)) return PyLong_FromLong(-1);
    const at::Tensor *W = plain(args[0]), *lut = plain(args[1]), *scales = plain(args[4]), *packed = plain(args[5]);
    if (!W || !lut || !scales || !packed) return PyLong_FromLong(-1);
    const int code = dtype_code(*lut);
    const bool f32 = W->scalar_type() == at::kFloat;
    if (code < 0 || (!f32 && dtype_code(*W) != code) || dtype_code(*scales) != code || W->dim() != 2) return PyLong_FromLong(-1);
    const int64_t N = W->size(0), K = W->size(1);
    if (!shape_is(*scales, N, K / group) || lut->numel() != (1 << bits) ||
        packed->numel() * packed->element_size() != (int64_t)packed_bytes(N, K, bits, group))
        return PyLong_FromLong(-1);
    const void *w = W->data_ptr(), *l = lut->data_ptr();
    void *s = scales->data_ptr(), *p = packed->data_ptr(), *stream = current_stream();
    lutq_status st;
    {
        WithoutGil released;
        st = quantize(w, f32 ? 1 : 0, l, bits, group, N, K, (lutq_dtype)code, s, p, stream);
    }
    return PyLong_FromLong((long)st);
}); }

// (packed, scales, lut, bits, group_size, W_out) -> status, or -1
PyObject* dequantise(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    int bits, group;
    if (!dequant || n != 6 || !small_int(args[3], 2, 4, &bits) || !small_int(args[4], 1, 1 << 16, &group)) return PyLong_FromLong(-1);
    const at::Tensor *packed = plain(args[0]), *scales = plain(args[1]), *lut = plain(args[2]), *W = plain(args[5]);
    if (!W || !lut || !scales || !packed) return PyLong_FromLong(-1);
    const int code = dtype_code(*W);
    if (code < 0 || dtype_code(*lut) != code || dtype_code(*scales) != code || W->dim() != 2 || scales->dim() != 2) return PyLong_FromLong(-1);
    const int64_t N = W->size(0), K = W->size(1);
    if (scales->size(0) != N || scales->size(1) * group != K || lut->numel() != (1 << bits) ||
        packed->numel() != (int64_t)packed_bytes(N, K, bits, group))
        return PyLong_FromLong(-1);
    const void *p = packed->data_ptr(), *s = scales->data_ptr(), *l = lut->data_ptr();
    void *w = W->data_ptr(), *stream = current_stream();
    lutq_status st;
    {
        WithoutGil released;
        st = dequant(p, s, l, bits, group, N, K, (lutq_dtype)code, w, stream);
    }
    return PyLong_FromLong((long)st);
}); }

// Whether `o` is None (then *t stays null) or a plain tensor.
bool plain_or_none(PyObject* o, const at::Tensor** t) {
    if (o == Py_None) return true;
    *t = plain(o);
    return *t != nullptr;
}

// Tensors (null ones aside) on the current device.  (The older calls leave the device to the caller.)
template <typename... T> bool on_current_device(const T*... t) {
    const auto here = c10::hip::current_device();
    return ((!t || t->get_device() == here) && ...);
}

bool is_bytes(const at::Tensor* t) { return !t || t->scalar_type() == at::kByte; }
bool is_numbers(const at::Tensor* t) { return !t || (t->scalar_type() == at::kInt && t->dim() == 1); }

// (X, codes, exponents or None for the packed form, rows or None) -> status, or -1
PyObject* mx4_quant(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    if (!mx4_quantize || n != 4) return PyLong_FromLong(-1);
    const at::Tensor *X = plain(args[0]), *codes = plain(args[1]), *exponents = nullptr, *rows = nullptr;
    if (!X || !codes || !plain_or_none(args[2], &exponents) || !plain_or_none(args[3], &rows) || X->dim() != 2 ||
        !on_current_device(X, codes, exponents, rows) || !is_bytes(codes) || !is_bytes(exponents) || !is_numbers(rows))
        return PyLong_FromLong(-1);
    const bool f32 = X->scalar_type() == at::kFloat;
    const int code = f32 ? LUTQ_F16 : dtype_code(*X);
    const int64_t from = X->size(0), K = X->size(1), M = rows ? rows->size(0) : from;
    if (code < 0) return PyLong_FromLong(-1);
    if (exponents ? K % 32 != 0 || !shape_is(*codes, M, K / 2) || !shape_is(*exponents, M, K / 32)
                  : rows || codes->numel() == 0 || codes->numel() != (int64_t)mx4_packed_bytes(M, K))
        return PyLong_FromLong(-1);
    const void *x = X->data_ptr(), *r = rows ? rows->data_ptr() : nullptr;
    void *c = codes->data_ptr(), *e = exponents ? exponents->data_ptr() : nullptr, *stream = current_stream();
    const lutq_dtype dt = (lutq_dtype)code;
    lutq_status st;
    {
        WithoutGil released;
        st = e || exponents ? mx4_quantize(x, f32, dt, from, static_cast<const int32_t*>(r), M, K, c, e, stream)
                            : mx4_quantize_packed(x, f32, dt, M, K, c, stream);
    }
    return PyLong_FromLong((long)st);
}); }

// (codes, exponents or None for the packed form, out) -> status, or -1
PyObject* mx4_dequantise(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    if (!mx4_dequant || n != 3) return PyLong_FromLong(-1);
    const at::Tensor *codes = plain(args[0]), *exponents = nullptr, *out = plain(args[2]);
    if (!codes || !plain_or_none(args[1], &exponents) || !out || out->dim() != 2 || !on_current_device(codes, exponents, out) ||
        !is_bytes(codes) || !is_bytes(exponents))
        return PyLong_FromLong(-1);
    const int code = dtype_code(*out);
    const int64_t M = out->size(0), K = out->size(1);
    if (code < 0) return PyLong_FromLong(-1);
    if (exponents ? K % 32 != 0 || !shape_is(*codes, M, K / 2) || !shape_is(*exponents, M, K / 32)
                  : codes->numel() == 0 || codes->numel() != (int64_t)mx4_packed_bytes(M, K))
        return PyLong_FromLong(-1);
    const void *c = codes->data_ptr(), *e = exponents ? exponents->data_ptr() : nullptr;
    void *w = out->data_ptr(), *stream = current_stream();
    lutq_status st;
    {
        WithoutGil released;
        st = exponents ? mx4_dequant(c, e, M, K, (lutq_dtype)code, w, stream) : mx4_dequant_packed(c, M, K, (lutq_dtype)code, w, stream);
    }
    return PyLong_FromLong((long)st);
}); }

// (X, exponents or None, packed, offsets or None, Y, workspace) -> status, or -1
PyObject* mx4_mm(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    if (!mx4_matmul || n != 6) return PyLong_FromLong(-1);
    const at::Tensor *X = plain(args[0]), *xe = nullptr, *packed = plain(args[2]), *offsets = nullptr, *Y = plain(args[4]), *ws = plain(args[5]);
    if (!X || !plain_or_none(args[1], &xe) || !packed || !plain_or_none(args[3], &offsets) || !Y || !ws || X->dim() != 2 || Y->dim() != 2 ||
        !on_current_device(X, xe, packed, offsets, Y, ws) || !is_bytes(xe) || !is_bytes(packed) || !is_bytes(ws) || !is_numbers(offsets))
        return PyLong_FromLong(-1);
    const int code = dtype_code(*Y);
    const int64_t M = Y->size(0), N = Y->size(1), K = X->size(1) * (xe ? 2 : 1), experts = offsets ? offsets->size(0) - 1 : 1;
    if (code < 0 || X->size(0) != M || (xe ? X->scalar_type() != at::kByte || K % 32 != 0 || !shape_is(*xe, M, K / 32)
                                           : X->scalar_type() != Y->scalar_type()))
        return PyLong_FromLong(-1);
    if (experts < 1 || packed->numel() == 0 || packed->numel() != experts * (int64_t)mx4_packed_bytes(N, K)) return PyLong_FromLong(-1);
    const void *x = X->data_ptr(), *e = xe ? xe->data_ptr() : nullptr, *w = packed->data_ptr(), *at = offsets ? offsets->data_ptr() : nullptr;
    void *y = Y->data_ptr(), *scratch = ws->data_ptr(), *stream = current_stream();
    const size_t bytes = (size_t)ws->numel();
    const lutq_dtype dt = (lutq_dtype)code;
    lutq_status st;
    {
        WithoutGil released;
        st = offsets ? mx4_matmul_grouped(x, e, w, static_cast<const int32_t*>(at), experts, M, N, K, dt, y, scratch, bytes, stream)
                     : mx4_matmul(x, e, w, M, N, K, dt, y, scratch, bytes, stream);
    }
    return PyLong_FromLong((long)st);
}); }

// ---- 8-bit floating point, blocks of 128
bool is_codes(const at::Tensor* t) { return !t || t->scalar_type() == at::kByte || t->scalar_type() == at::kFloat8_e4m3fn; }
bool is_scales(const at::Tensor* t) { return !t || t->scalar_type() == at::kFloat; }
bool fits(const at::Tensor* t, int64_t a, int64_t b) { return !t || shape_is(*t, a, b); }
int64_t up128(int64_t n) { return (n + 127) / 128; }
void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
float* floats(const at::Tensor* t) { return static_cast<float*>(data(t)); }

enum QuantiseKind { kRows = 0, kWeights = 1, kColumns = 2 };

// (kind, X, codes, scales, rows or None, transposed codes or None, transposed scales or None) -> status, or -1
PyObject* fp8_quant(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    int kind;
    if (!fp8_quantize || n != 7 || !small_int(args[0], 0, 2, &kind)) return PyLong_FromLong(-1);
    const at::Tensor *X = plain(args[1]), *codes = plain(args[2]), *scales = plain(args[3]), *rows = nullptr, *t = nullptr, *ts = nullptr;
    if (!X || !codes || !scales || !plain_or_none(args[4], &rows) || !plain_or_none(args[5], &t) || !plain_or_none(args[6], &ts) || X->dim() != 2 ||
        !on_current_device(X, codes, scales, rows, t, ts) || !is_codes(codes) || !is_codes(t) || !is_scales(scales) || !is_scales(ts) || !is_numbers(rows) || !t != !ts)
        return PyLong_FromLong(-1);
    const bool f32 = X->scalar_type() == at::kFloat;
    const int code = f32 ? LUTQ_F16 : dtype_code(*X);
    const int64_t from = X->size(0), K = X->size(1), M = rows ? rows->size(0) : from;
    if (code < 0 || (kind == kRows      ? !shape_is(*codes, M, K) || !shape_is(*scales, K / 128, M)
                     : kind == kWeights ? !shape_is(*codes, M, K) || !shape_is(*scales, up128(M), K / 128) || !fits(t, K, M) || !fits(ts, K / 128, up128(M))
                                        : !shape_is(*codes, K, 128 * up128(M)) || !shape_is(*scales, up128(M), K)))
        return PyLong_FromLong(-1);
    const void *x = data(X), *r = data(rows);
    void *c = data(codes), *tc = data(t), *stream = current_stream();
    float *s = floats(scales), *tcs = floats(ts);
    const lutq_dtype dt = (lutq_dtype)code;
    lutq_status st;
    {
        WithoutGil released;
        st = kind == kRows      ? fp8_quantize(x, f32, dt, from, static_cast<const int32_t*>(r), M, K, c, s, stream)
             : kind == kWeights ? fp8_quantize_weights(x, f32, dt, M, K, c, s, tc, tcs, stream)
                                : fp8_quantize_columns(x, f32, dt, M, K, c, s, stream);
    }
    return PyLong_FromLong((long)st);
}); }

// (kind, codes, scales, out) -> status, or -1
PyObject* fp8_dequantise(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    int kind;
    if (!fp8_dequant || n != 4 || !small_int(args[0], 0, 1, &kind)) return PyLong_FromLong(-1);
    const at::Tensor *codes = plain(args[1]), *scales = plain(args[2]), *out = plain(args[3]);
    if (!codes || !scales || !out || out->dim() != 2 || !on_current_device(codes, scales, out) || !is_codes(codes) || !is_scales(scales)) return PyLong_FromLong(-1);
    const int code = dtype_code(*out);
    const int64_t M = out->size(0), K = out->size(1);
    if (code < 0 || !shape_is(*codes, M, K) || !(kind == kRows ? shape_is(*scales, K / 128, M) : shape_is(*scales, up128(M), K / 128))) return PyLong_FromLong(-1);
    const void* c = data(codes);
    const float* s = floats(scales);
    void *w = data(out), *stream = current_stream();
    lutq_status st;
    {
        WithoutGil released;
        st = (kind == kRows ? fp8_dequant : fp8_dequant_weights)(c, s, M, K, (lutq_dtype)code, w, stream);
    }
    return PyLong_FromLong((long)st);
}); }

bool is_weights(const at::Tensor& W, const at::Tensor& ws, int64_t experts, int64_t N, int64_t K) {
    if (experts < 0) return shape_is(W, N, K) && shape_is(ws, up128(N), K / 128);
    return W.dim() == 3 && ws.dim() == 3 && W.size(0) == experts && W.size(1) == N && W.size(2) == K && ws.size(0) == experts && ws.size(1) == up128(N) && ws.size(2) == K / 128;
}

// (X, scales or None, W, scales, offsets or None, activation or -1 for the plain product, 0 or 1 for H's dtype, Y or None, codes of H or None, their
// scales or None, saved or None, workspace) -> status, or -1
PyObject* fp8_mm(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    int act, code;
    if (!fp8_matmul || n != 12 || !small_int(args[5], -1, 1, &act) || !small_int(args[6], 0, 1, &code)) return PyLong_FromLong(-1);
    const at::Tensor *X = plain(args[0]), *xs = nullptr, *W = plain(args[2]), *ws = plain(args[3]), *offsets = nullptr, *Y = nullptr, *hc = nullptr,
                     *hs = nullptr, *saved = nullptr, *work = plain(args[11]);
    if (!X || !plain_or_none(args[1], &xs) || !W || !ws || !plain_or_none(args[4], &offsets) || !plain_or_none(args[7], &Y) || !plain_or_none(args[8], &hc) ||
        !plain_or_none(args[9], &hs) || !plain_or_none(args[10], &saved) || !work || (!Y && !hc) || !hc != !hs || X->dim() != 2 ||
        !on_current_device(X, xs, W, ws, offsets, Y, hc, hs, saved, work))
        return PyLong_FromLong(-1);
    const at::Tensor& out = Y ? *Y : *hc;
    if (out.dim() != 2 || (xs && !is_codes(X)) || (!xs && dtype_code(*X) != code) || !is_codes(W) || !is_codes(hc) || !is_scales(xs) || !is_scales(ws) || !is_scales(hs) ||
        !is_bytes(work) || !is_numbers(offsets) || (Y && dtype_code(*Y) != code) || (saved && dtype_code(*saved) != code))
        return PyLong_FromLong(-1);
    const int64_t M = out.size(0), N = out.size(1), K = X->size(1), rows = act < 0 ? N : 2 * N, experts = offsets ? offsets->size(0) - 1 : -1;
    if ((act < 0 && (hc || saved)) || (offsets && experts < 1) || X->size(0) != M || !fits(xs, K / 128, M) || !is_weights(*W, *ws, experts, rows, K) ||
        !fits(hc, M, N) || !fits(hs, N / 128, M) || !fits(saved, M, 2 * N))
        return PyLong_FromLong(-1);
    const void *x = data(X), *w = data(W);
    const float *xf = floats(xs), *wf = floats(ws);
    const int32_t* at = static_cast<const int32_t*>(data(offsets));
    void *y = data(Y), *h = data(hc), *sv = data(saved), *scratch = data(work), *stream = current_stream();
    float* hf = floats(hs);
    const size_t bytes = (size_t)work->numel();
    const lutq_dtype dt = (lutq_dtype)code;
    lutq_status st;
    {
        WithoutGil released;
        st = act < 0 ? (at ? fp8_matmul_grouped(x, xf, w, wf, at, experts, M, N, K, dt, y, scratch, bytes, stream)
                           : fp8_matmul(x, xf, w, wf, M, N, K, dt, y, scratch, bytes, stream))
                     : (at ? fp8_gated_grouped(x, xf, w, wf, at, experts, M, N, K, (lutq_activation)act, dt, y, h, hf, sv, scratch, bytes, stream)
                           : fp8_gated(x, xf, w, wf, M, N, K, (lutq_activation)act, dt, y, h, hf, sv, scratch, bytes, stream));
    }
    return PyLong_FromLong((long)st);
}); }

// (dH, saved, activation, dense or None, row codes or None, their scales or None, column codes or None, their scales or None) -> status, or -1
PyObject* fp8_grad(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    int act;
    if (!fp8_gated_grad || n != 8 || !small_int(args[2], 0, 1, &act)) return PyLong_FromLong(-1);
    const at::Tensor *dh = plain(args[0]), *saved = plain(args[1]), *dense = nullptr, *rc = nullptr, *rs = nullptr, *cc = nullptr, *cs = nullptr;
    if (!dh || !saved || !plain_or_none(args[3], &dense) || !plain_or_none(args[4], &rc) || !plain_or_none(args[5], &rs) || !plain_or_none(args[6], &cc) ||
        !plain_or_none(args[7], &cs) || dh->dim() != 2 || !on_current_device(dh, saved, dense, rc, rs, cc, cs))
        return PyLong_FromLong(-1);
    const int code = dtype_code(*dh);
    const int64_t M = dh->size(0), F = dh->size(1);
    if (code < 0 || dtype_code(*saved) != code || (dense && dtype_code(*dense) != code) || !is_codes(rc) || !is_codes(cc) || !is_scales(rs) || !is_scales(cs) ||
        (!dense && !rc && !cc) || !rc != !rs || !cc != !cs || !shape_is(*saved, M, 2 * F) || !fits(dense, M, 2 * F) || !fits(rc, M, 2 * F) || !fits(rs, 2 * F / 128, M) ||
        !fits(cc, 2 * F, 128 * up128(M)) || !fits(cs, up128(M), 2 * F))
        return PyLong_FromLong(-1);
    const void *d = data(dh), *s = data(saved);
    void *out = data(dense), *r = data(rc), *c = data(cc), *stream = current_stream();
    float *rf = floats(rs), *cf = floats(cs);
    lutq_status st;
    {
        WithoutGil released;
        st = fp8_gated_grad(d, s, M, F, (lutq_activation)act, (lutq_dtype)code, out, r, rf, c, cf, stream);
    }
    return PyLong_FromLong((long)st);
}); }

// (dY, scales, X, scales, dW, workspace) -> status, or -1
PyObject* fp8_wgrad(PyObject*, PyObject* const* args, Py_ssize_t n) { return answer([&]() -> PyObject* {
    if (!fp8_weight_grad || n != 6) return PyLong_FromLong(-1);
    const at::Tensor *dy = plain(args[0]), *ds = plain(args[1]), *X = plain(args[2]), *xs = plain(args[3]), *dw = plain(args[4]), *work = plain(args[5]);
    if (!dy || !ds || !X || !xs || !dw || !work || dy->dim() != 2 || dw->dim() != 2 || !on_current_device(dy, ds, X, xs, dw, work) || !is_codes(dy) || !is_codes(X) ||
        !is_scales(ds) || !is_scales(xs) || !is_bytes(work))
        return PyLong_FromLong(-1);
    const int code = dtype_code(*dw);
    const int64_t N = dw->size(0), K = dw->size(1), M = dy->size(1);
    if (code < 0 || !shape_is(*dy, N, M) || !shape_is(*ds, M / 128, N) || !shape_is(*X, K, M) || !shape_is(*xs, M / 128, K)) return PyLong_FromLong(-1);
    const void *d = data(dy), *x = data(X);
    const float *df = floats(ds), *xf = floats(xs);
    void *w = data(dw), *scratch = data(work), *stream = current_stream();
    const size_t bytes = (size_t)work->numel();
    lutq_status st;
    {
        WithoutGil released;
        st = fp8_weight_grad(d, df, x, xf, N, K, M, (lutq_dtype)code, w, scratch, bytes, stream);
    }
    return PyLong_FromLong((long)st);
}); }

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, nullptr},
    {"mm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mm)), METH_FASTCALL, nullptr},
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quant)), METH_FASTCALL, nullptr},
    {"dequant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(dequantise)), METH_FASTCALL, nullptr},
    {"mx4_quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx4_quant)), METH_FASTCALL, nullptr},
    {"mx4_dequant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx4_dequantise)), METH_FASTCALL, nullptr},
    {"mx4_mm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx4_mm)), METH_FASTCALL, nullptr},
    {"fp8_quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp8_quant)), METH_FASTCALL, nullptr},
    {"fp8_dequant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp8_dequantise)), METH_FASTCALL, nullptr},
    {"fp8_mm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp8_mm)), METH_FASTCALL, nullptr},
    {"fp8_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp8_grad)), METH_FASTCALL, nullptr},
    {"fp8_weight_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp8_wgrad)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lutq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lutq_torch() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", LUTQ_TORCH_VERSION) != 0) { Py_DECREF(m); return nullptr; }
    return m;
}
