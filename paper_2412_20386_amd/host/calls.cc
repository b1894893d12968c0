// The per-call half of the Python binding in C++: the launches of the hot path as Python callables.
//
// A pass over a small layer is a handful of kernels of 3 - 6 us, and marshalled through ctypes a call took 9 - 10 us of
// host time (argument checks 4, conversion of the C arguments 2, current stream 1.3, launch 2 - 3), so small batches ran at
// the speed of the interpreter.  The same checks, in the same order and with the same messages, take well under a
// microsecond here.  No arithmetic, no allocation but the outputs that the caller leaves out, no state but the table
// of entry points, which is filled once from the loaded libptq4vm.so.
#include <ATen/ATen.h>
#include <Python.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/ptq4vm.h"

namespace {

struct Raised {};  // a Python exception is set

[[noreturn]] void raise(PyObject *type, const std::string &text) {
    PyErr_SetString(type, text.c_str());
    throw Raised{};
}

// ---------------------------------------------------------------------------------- entry points of the library
#define PTQ4VM_HOT_ENTRIES(X)                                                                                      \
    X(quantize_pts) X(quantize_dynamic) X(quantize_pts_offset) X(quantize_pts_a4) X(quantize_pts_a4_e2m3)          \
    X(w8a8_linear) X(w8a8_linear_offset) X(w4a4_linear) X(w4a4_linear_e2m3) X(w8a8_linear_fused)                   \
    X(w8a8_linear_offset_fused) X(w4a4_linear_fused) X(f16_linear)                                                 \
    X(gated_scan) X(gated_scan_workspace) X(gated_scan_backward) X(gated_scan_backward_workspace) X(gated_scan_step) \
    X(token_conv) X(token_conv_backward) X(token_conv_backward_workspace) X(token_conv_step) X(residual_norm)      \
    X(residual_norm_backward) X(residual_norm_backward_workspace)

struct Entries {
#define X(name) decltype(&ptq4vm_##name) name = nullptr;
    PTQ4VM_HOT_ENTRIES(X)
#undef X
} entry;
bool bound = false;
PyObject *load_library = nullptr;  // binding._load_entries(): calls bind() below, raises if the library is missing
PyObject *raise_status = nullptr;  // binding.check(status)

void need_library() {
    if (bound) return;
    PyObject *r = PyObject_CallNoArgs(load_library);
    if (!r) throw Raised{};
    Py_DECREF(r);
}

void check(int status) {
    if (status == PTQ4VM_OK) return;
    PyObject *r = PyObject_CallFunction(raise_status, "i", status);
    Py_XDECREF(r);
    throw Raised{};
}

// Calls f(current stream) without the interpreter lock (a launch waits when its queue is full) and raises for its status.
template <typename F>
void launch(F &&f) {
    void *const stream = static_cast<void *>(c10::hip::getCurrentHIPStream().stream());
    PyThreadState *const state = PyEval_SaveThread();
    const int status = f(stream);
    PyEval_RestoreThread(state);
    check(status);
}

// ---------------------------------------------------------------------------------- arguments
const char *dtype_name(at::ScalarType t) {
    switch (t) {
        case at::kHalf: return "torch.float16";
        case at::kBFloat16: return "torch.bfloat16";
        case at::kChar: return "torch.int8";
        case at::kByte: return "torch.uint8";
        case at::kInt: return "torch.int32";
        default: return "torch.float32";
    }
}

bool given(PyObject *o) { return o && o != Py_None; }

const at::Tensor *tensor(PyObject *o) { return o && THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

struct Matrix {
    int64_t rows, cols, ld;
    void *data;
};

Matrix matrix(PyObject *o, at::ScalarType dtype, const char *name) {
    const at::Tensor *t = tensor(o);
    if (!t || !t->is_cuda() || t->scalar_type() != dtype || t->dim() != 2 || (t->size(1) > 1 && t->stride(1) != 1))
        raise(PyExc_TypeError, std::string(name) + ": expected a 2-D CUDA tensor of " + dtype_name(dtype) + " with unit inner stride");
    const int64_t rows = t->size(0), cols = t->size(1), pitch = t->stride(0);
    return {rows, cols, rows > 1 ? pitch : std::max(pitch, cols), t->data_ptr()};
}

// A matrix that the kernels write rows x cols elements of.  A larger one (a buffer of the largest batch) is taken too; the
// C boundary sees a pointer and a pitch only, so a smaller one has to be refused here.
Matrix written(PyObject *o, at::ScalarType dtype, int64_t rows, int64_t cols, const char *name) {
    const Matrix m = matrix(o, dtype, name);
    if (m.rows < rows || m.cols < cols)
        raise(PyExc_ValueError, std::string(name) + ": expected at least " + std::to_string(rows) + " x " + std::to_string(cols) + " elements, got " +
                                    std::to_string(m.rows) + " x " + std::to_string(m.cols));
    return m;
}

void *vector(PyObject *o, at::ScalarType dtype, int64_t n, const char *name, bool optional = false) {
    if (!given(o)) {
        if (optional) return nullptr;
        raise(PyExc_TypeError, std::string(name) + " is required");
    }
    const at::Tensor *t = tensor(o);
    if (!t || !t->is_cuda() || t->scalar_type() != dtype || t->dim() != 1 || t->size(0) != n || !t->is_contiguous())
        raise(PyExc_TypeError, std::string(name) + ": expected a contiguous CUDA vector of " + std::to_string(n) + " x " + dtype_name(dtype));
    return t->data_ptr();
}

void *accumulators(PyObject *o, int64_t M, int64_t N) {
    if (!given(o)) return nullptr;
    const at::Tensor *t = tensor(o);
    if (!t || !t->is_cuda() || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != M || t->size(1) != N || !t->is_contiguous())
        raise(PyExc_TypeError, "acc_out: expected a dense CUDA int32 [M, N] tensor");
    return t->data_ptr();
}

int64_t integer(PyObject *o) {
    const int64_t v = PyLong_Check(o) ? PyLong_AsLongLong(o) : [&] {
        PyObject *i = PyNumber_Index(o);
        if (!i) throw Raised{};
        const int64_t w = PyLong_AsLongLong(i);
        Py_DECREF(i);
        return w;
    }();
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

int64_t e2m3_blocks(int64_t K) { return (K + 127) / 128; }

struct Container {
    int64_t pitch;
    void *data;
};

Container container(PyObject *o, int64_t rows, int64_t K, const char *name) {
    const at::Tensor *t = tensor(o);
    if (!t || !t->is_cuda() || t->scalar_type() != at::kByte || t->dim() != 3)
        raise(PyExc_TypeError, std::string(name) + ": expected a CUDA uint8 tensor [blocks, rows, 96]");
    const int64_t blocks = e2m3_blocks(K);
    if (t->size(0) != blocks || t->size(1) != rows || t->size(2) != 96 || t->stride(2) != 1 || (rows > 1 && t->stride(1) != 96))
        raise(PyExc_ValueError, std::string(name) + ": expected shape (" + std::to_string(blocks) + ", " + std::to_string(rows) +
                                    ", 96) with dense 96-byte blocks");
    return {blocks > 1 ? t->stride(0) : std::max<int64_t>(t->stride(0), 96 * rows), t->data_ptr()};
}

// An output: the caller's tensor (a new reference to it) or a fresh one on the device of `like`.
PyObject *output(PyObject *o, at::IntArrayRef shape, at::ScalarType dtype, PyObject *like) {
    if (given(o)) {
        Py_INCREF(o);
        return o;
    }
    PyObject *w = THPVariable_Wrap(at::empty(shape, THPVariable_Unpack(like).options().dtype(dtype)));
    if (!w) throw Raised{};
    return w;
}

struct Owned {  // releases the output when a later step raises
    PyObject *o;
    explicit Owned(PyObject *p) : o(p) {}
    Owned(const Owned &) = delete;
    ~Owned() { Py_XDECREF(o); }
    PyObject *release() {
        PyObject *p = o;
        o = nullptr;
        return p;
    }
};

const float *floats(void *p) { return static_cast<const float *>(p); }
const int8_t *codes(const Matrix &m) { return static_cast<const int8_t *>(m.data); }
const uint8_t *bytes(void *p) { return static_cast<const uint8_t *>(p); }
const int32_t *ints(void *p) { return static_cast<const int32_t *>(p); }

// M == B * L, in exact arithmetic
bool is_product(int64_t M, int64_t B, int64_t L) {
    int64_t p;
    return !__builtin_mul_overflow(B, L, &p) && p == M;
}
void same_rows(int64_t M, int64_t B, int64_t L) {
    if (!is_product(M, B, L)) raise(PyExc_ValueError, "x must have B*L rows");
}
void same_shape(bool ok) {
    if (!ok) raise(PyExc_ValueError, "shape mismatch");
}

// ---------------------------------------------------------------------------------- the calls
using Args = PyObject *const *;

PyObject *quantize_pts(Args a) {  // x inv_m s_tok B L xq
    const Matrix x = matrix(a[0], at::kHalf, "x");
    const int64_t B = integer(a[3]), L = integer(a[4]);
    same_rows(x.rows, B, L);
    void *inv_m = vector(a[1], at::kFloat, x.cols, "inv_m", true), *s_tok = vector(a[2], at::kFloat, L, "s_tok");
    Owned out(output(a[5], {x.rows, x.cols}, at::kChar, a[0]));
    const Matrix xq = written(out.o, at::kChar, x.rows, x.cols, "xq");
    launch([&](void *s) { return entry.quantize_pts(x.data, floats(inv_m), floats(s_tok), static_cast<int8_t *>(xq.data), B, L, x.cols, x.ld, xq.ld, s); });
    return out.release();
}

PyObject *quantize_pts_offset(Args a) {  // x inv_m s_tok z_tok B L xq
    const Matrix x = matrix(a[0], at::kHalf, "x");
    const int64_t B = integer(a[4]), L = integer(a[5]);
    same_rows(x.rows, B, L);
    void *inv_m = vector(a[1], at::kFloat, x.cols, "inv_m", true), *s_tok = vector(a[2], at::kFloat, L, "s_tok"),
         *z_tok = vector(a[3], at::kInt, L, "z_tok");
    Owned out(output(a[6], {x.rows, x.cols}, at::kChar, a[0]));
    const Matrix xq = written(out.o, at::kChar, x.rows, x.cols, "xq");
    launch([&](void *s) { return entry.quantize_pts_offset(x.data, floats(inv_m), floats(s_tok), ints(z_tok), static_cast<int8_t *>(xq.data), B, L, x.cols,
                                    x.ld, xq.ld, s); });
    return out.release();
}

PyObject *quantize_pts_a4(Args a) {  // x inv_m s_tok B L xq4
    const Matrix x = matrix(a[0], at::kHalf, "x");
    const int64_t B = integer(a[3]), L = integer(a[4]);
    same_rows(x.rows, B, L);
    void *inv_m = vector(a[1], at::kFloat, x.cols, "inv_m", true), *s_tok = vector(a[2], at::kFloat, L, "s_tok");
    Owned out(output(a[5], {x.rows, x.cols / 2}, at::kByte, a[0]));
    const Matrix xq = written(out.o, at::kByte, x.rows, x.cols / 2, "xq4");
    launch([&](void *s) { return entry.quantize_pts_a4(x.data, floats(inv_m), floats(s_tok), static_cast<uint8_t *>(xq.data), B, L, x.cols, x.ld, xq.ld, s); });
    return out.release();
}

PyObject *quantize_pts_a4_e2m3(Args a) {  // x inv_m s_tok B L xq6
    const Matrix x = matrix(a[0], at::kHalf, "x");
    const int64_t B = integer(a[3]), L = integer(a[4]);
    same_rows(x.rows, B, L);
    void *inv_m = vector(a[1], at::kFloat, x.cols, "inv_m", true), *s_tok = vector(a[2], at::kFloat, L, "s_tok");
    Owned out(output(a[5], {e2m3_blocks(x.cols), x.rows, 96}, at::kByte, a[0]));
    const Container xq = container(out.o, x.rows, x.cols, "xq6");
    launch([&](void *s) { return entry.quantize_pts_a4_e2m3(x.data, floats(inv_m), floats(s_tok), static_cast<uint8_t *>(xq.data), B, L, x.cols, x.ld, xq.pitch,
                                     s); });
    return out.release();
}

PyObject *quantize_dynamic(Args a) {  // x inv_m xq s_row
    const Matrix x = matrix(a[0], at::kHalf, "x");
    void *inv_m = vector(a[1], at::kFloat, x.cols, "inv_m", true);
    Owned out(output(a[2], {x.rows, x.cols}, at::kChar, a[0]));
    const Matrix xq = written(out.o, at::kChar, x.rows, x.cols, "xq");
    Owned steps(output(a[3], {x.rows}, at::kFloat, a[0]));
    void *s_row = vector(steps.o, at::kFloat, x.rows, "s_row");
    launch([&](void *s) { return entry.quantize_dynamic(x.data, floats(inv_m), static_cast<int8_t *>(xq.data), static_cast<float *>(s_row), x.rows, x.cols, x.ld,
                                 xq.ld, s); });
    PyObject *pair = PyTuple_Pack(2, out.o, steps.o);
    if (!pair) throw Raised{};
    return pair;
}

PyObject *w8a8_linear(Args a) {  // xq wq s_tok s_w bias B L y acc_out
    const Matrix xq = matrix(a[0], at::kChar, "xq"), wq = matrix(a[1], at::kChar, "wq");
    const int64_t B = integer(a[5]), L = integer(a[6]), M = xq.rows, N = wq.rows;
    same_shape(xq.cols == wq.cols && is_product(M, B, L));
    void *s_tok = vector(a[2], at::kFloat, L, "s_tok"), *s_w = vector(a[3], at::kFloat, N, "s_w"), *bias = vector(a[4], at::kHalf, N, "bias", true);
    Owned out(output(a[7], {M, N}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, M, N, "y");
    void *acc = accumulators(a[8], M, N);
    launch([&](void *s) { return entry.w8a8_linear(codes(xq), codes(wq), floats(s_tok), floats(s_w), bias, y.data, static_cast<int32_t *>(acc), B, L, xq.cols, N,
                            xq.ld, wq.ld, y.ld, s); });
    return out.release();
}

PyObject *w8a8_linear_offset(Args a) {  // xq wq s_tok z_tok rowsum s_w bias B L y acc_out
    const Matrix xq = matrix(a[0], at::kChar, "xq"), wq = matrix(a[1], at::kChar, "wq");
    const int64_t B = integer(a[7]), L = integer(a[8]), M = xq.rows, N = wq.rows;
    same_shape(xq.cols == wq.cols && is_product(M, B, L));
    void *s_tok = vector(a[2], at::kFloat, L, "s_tok"), *z_tok = vector(a[3], at::kInt, L, "z_tok"),
         *rowsum = vector(a[4], at::kInt, N, "rowsum"), *s_w = vector(a[5], at::kFloat, N, "s_w"),
         *bias = vector(a[6], at::kHalf, N, "bias", true);
    Owned out(output(a[9], {M, N}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, M, N, "y");
    void *acc = accumulators(a[10], M, N);
    launch([&](void *s) { return entry.w8a8_linear_offset(codes(xq), codes(wq), floats(s_tok), ints(z_tok), ints(rowsum), floats(s_w), bias, y.data,
                                   static_cast<int32_t *>(acc), B, L, xq.cols, N, xq.ld, wq.ld, y.ld, s); });
    return out.release();
}

PyObject *w4a4_linear(Args a) {  // xq4 wq4 s_tok s_w bias B L y acc_out
    const Matrix xq = matrix(a[0], at::kByte, "xq4"), wq = matrix(a[1], at::kByte, "wq4");
    const int64_t B = integer(a[5]), L = integer(a[6]), M = xq.rows, N = wq.rows;
    same_shape(xq.cols == wq.cols && is_product(M, B, L));
    void *s_tok = vector(a[2], at::kFloat, L, "s_tok"), *s_w = vector(a[3], at::kFloat, N, "s_w"), *bias = vector(a[4], at::kHalf, N, "bias", true);
    Owned out(output(a[7], {M, N}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, M, N, "y");
    void *acc = accumulators(a[8], M, N);
    launch([&](void *s) { return entry.w4a4_linear(bytes(xq.data), bytes(wq.data), floats(s_tok), floats(s_w), bias, y.data, static_cast<int32_t *>(acc), B, L,
                            2 * xq.cols, N, xq.ld, wq.ld, y.ld, s); });
    return out.release();
}

PyObject *w4a4_linear_e2m3(Args a) {  // xq6 wq6 s_tok s_w bias B L K y acc_out
    const int64_t B = integer(a[5]), L = integer(a[6]), K = integer(a[7]);
    int64_t M;
    if (__builtin_mul_overflow(B, L, &M)) raise(PyExc_ValueError, "xq6: B*L is out of range");
    const Container xq = container(a[0], M, K, "xq6");
    const at::Tensor *w = tensor(a[1]);
    if (!w || w->dim() != 3) raise(PyExc_TypeError, "wq6: expected a CUDA uint8 tensor [blocks, N, 96]");
    const int64_t N = w->size(1);
    const Container wq = container(a[1], N, K, "wq6");
    void *s_tok = vector(a[2], at::kFloat, L, "s_tok"), *s_w = vector(a[3], at::kFloat, N, "s_w"), *bias = vector(a[4], at::kHalf, N, "bias", true);
    Owned out(output(a[8], {M, N}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, M, N, "y");
    void *acc = accumulators(a[9], M, N);
    launch([&](void *s) { return entry.w4a4_linear_e2m3(bytes(xq.data), bytes(wq.data), floats(s_tok), floats(s_w), bias, y.data, static_cast<int32_t *>(acc), B, L,
                                 K, N, xq.pitch, wq.pitch, y.ld, s); });
    return out.release();
}

struct CodesOut {
    int64_t ld = 0;
    int8_t *data = nullptr;
};
CodesOut codes_out(PyObject *o, int64_t M, int64_t K) {
    if (!given(o)) return {};
    const Matrix m = matrix(o, at::kChar, "xq_out");
    if (m.rows != M || m.cols != K) raise(PyExc_ValueError, "xq_out must be [B*L, K]");
    return {m.ld, static_cast<int8_t *>(m.data)};
}

PyObject *w8a8_linear_fused(Args a) {  // x inv_m s_tok wq s_w bias B L y acc_out xq_out
    const Matrix x = matrix(a[0], at::kHalf, "x"), wq = matrix(a[3], at::kChar, "wq");
    const int64_t B = integer(a[6]), L = integer(a[7]), M = x.rows, K = x.cols, N = wq.rows;
    same_shape(K == wq.cols && is_product(M, B, L));
    void *inv_m = vector(a[1], at::kFloat, K, "inv_m", true), *s_tok = vector(a[2], at::kFloat, L, "s_tok"),
         *s_w = vector(a[4], at::kFloat, N, "s_w"), *bias = vector(a[5], at::kHalf, N, "bias", true);
    Owned out(output(a[8], {M, N}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, M, N, "y");
    void *acc = accumulators(a[9], M, N);
    const CodesOut xq = codes_out(a[10], M, K);
    launch([&](void *s) { return entry.w8a8_linear_fused(x.data, floats(inv_m), floats(s_tok), codes(wq), floats(s_w), bias, y.data, static_cast<int32_t *>(acc),
                                  xq.data, B, L, K, N, x.ld, wq.ld, y.ld, xq.ld, s); });
    return out.release();
}

PyObject *w8a8_linear_offset_fused(Args a) {  // x inv_m s_tok z_tok wq rowsum s_w bias B L y acc_out xq_out
    const Matrix x = matrix(a[0], at::kHalf, "x"), wq = matrix(a[4], at::kChar, "wq");
    const int64_t B = integer(a[8]), L = integer(a[9]), M = x.rows, K = x.cols, N = wq.rows;
    same_shape(K == wq.cols && is_product(M, B, L));
    void *inv_m = vector(a[1], at::kFloat, K, "inv_m", true), *s_tok = vector(a[2], at::kFloat, L, "s_tok"),
         *z_tok = vector(a[3], at::kInt, L, "z_tok"), *rowsum = vector(a[5], at::kInt, N, "rowsum"),
         *s_w = vector(a[6], at::kFloat, N, "s_w"), *bias = vector(a[7], at::kHalf, N, "bias", true);
    Owned out(output(a[10], {M, N}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, M, N, "y");
    void *acc = accumulators(a[11], M, N);
    const CodesOut xq = codes_out(a[12], M, K);
    launch([&](void *s) { return entry.w8a8_linear_offset_fused(x.data, floats(inv_m), floats(s_tok), ints(z_tok), codes(wq), ints(rowsum), floats(s_w), bias, y.data,
                                         static_cast<int32_t *>(acc), xq.data, B, L, K, N, x.ld, wq.ld, y.ld, xq.ld, s); });
    return out.release();
}

PyObject *w4a4_linear_fused(Args a) {  // x inv_m s_tok wq4 s_w bias B L y acc_out xq_out
    const Matrix x = matrix(a[0], at::kHalf, "x"), wq = matrix(a[3], at::kByte, "wq4");
    const int64_t B = integer(a[6]), L = integer(a[7]), M = x.rows, K = x.cols, N = wq.rows;
    same_shape(K == 2 * wq.cols && is_product(M, B, L));
    void *inv_m = vector(a[1], at::kFloat, K, "inv_m", true), *s_tok = vector(a[2], at::kFloat, L, "s_tok"),
         *s_w = vector(a[4], at::kFloat, N, "s_w"), *bias = vector(a[5], at::kHalf, N, "bias", true);
    Owned out(output(a[8], {M, N}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, M, N, "y");
    void *acc = accumulators(a[9], M, N);
    const CodesOut xq = codes_out(a[10], M, K);
    launch([&](void *s) { return entry.w4a4_linear_fused(x.data, floats(inv_m), floats(s_tok), bytes(wq.data), floats(s_w), bias, y.data, static_cast<int32_t *>(acc),
                                  xq.data, B, L, K, N, x.ld, wq.ld, y.ld, xq.ld, s); });
    return out.release();
}

PyObject *f16_linear(Args a) {  // x w bias y
    const Matrix x = matrix(a[0], at::kHalf, "x"), w = matrix(a[1], at::kHalf, "w");
    same_shape(x.cols == w.cols);
    void *bias = vector(a[2], at::kHalf, w.rows, "bias", true);
    Owned out(output(a[3], {x.rows, w.rows}, at::kHalf, a[0]));
    const Matrix y = written(out.o, at::kHalf, x.rows, w.rows, "y");
    launch([&](void *s) { return entry.f16_linear(x.data, w.data, bias, y.data, x.rows, x.cols, w.rows, x.ld, w.ld, y.ld, s); });
    return out.release();
}

// ---------------------------------------------------------------------------------- the operators between a block's linears
// Their tensors have to be on one device, which need not be the current one: the call goes to that device's current stream.
struct Operands {
    at::ScalarType dtype;  // T of the first one
    int code;              // its ptq4vm_dtype
    at::Device device;

    static const at::Tensor &first(PyObject *o, const char *name) {
        const at::Tensor *t = tensor(o);
        if (!t || !t->is_cuda() || (t->scalar_type() != at::kHalf && t->scalar_type() != at::kBFloat16 && t->scalar_type() != at::kFloat))
            raise(PyExc_TypeError, std::string(name) + ": expected a 2-D CUDA tensor of torch.float16, torch.bfloat16 or torch.float32");
        return *t;
    }
    static int code_of(at::ScalarType t) { return t == at::kHalf ? PTQ4VM_F16 : t == at::kBFloat16 ? PTQ4VM_BF16 : PTQ4VM_F32; }
    Operands(PyObject *o, const char *name) : dtype(first(o, name).scalar_type()), code(code_of(dtype)), device(first(o, name).device()) {}

    void here(PyObject *o, const char *name) const {
        if (THPVariable_Unpack(o).device() != device) raise(PyExc_ValueError, std::string(name) + ": on another device than the first operand");
    }
    // [rows, cols] of T (or `type`)
    Matrix in(PyObject *o, int64_t rows, int64_t cols, const char *name) const { return in(o, dtype, rows, cols, name); }
    Matrix in(PyObject *o, at::ScalarType type, int64_t rows, int64_t cols, const char *name) const {
        const Matrix m = matrix(o, type, name);
        here(o, name);
        if (m.rows != rows || m.cols != cols)
            raise(PyExc_ValueError, std::string(name) + ": expected " + std::to_string(rows) + " x " + std::to_string(cols) + " elements, got " + std::to_string(m.rows) +
                                        " x " + std::to_string(m.cols));
        return m;
    }
    Matrix optional(PyObject *o, at::ScalarType type, int64_t rows, int64_t cols, const char *name) const {
        return given(o) ? in(o, type, rows, cols, name) : Matrix{rows, cols, cols, nullptr};
    }
    Matrix out(PyObject *o, at::ScalarType type, int64_t rows, int64_t cols, const char *name) const {
        const Matrix m = written(o, type, rows, cols, name);
        here(o, name);
        return m;
    }
    const float *floats(PyObject *o, int64_t n, const char *name, bool optional = false) const {
        void *p = vector(o, at::kFloat, n, name, optional);
        if (p || given(o)) here(o, name);
        return static_cast<const float *>(p);
    }
    void *dense(PyObject *o, at::ScalarType type, at::IntArrayRef shape, const char *name) const {
        const at::Tensor *t = tensor(o);
        if (!t || !t->is_cuda() || t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous()) {
            std::string s;
            for (const int64_t n : shape) s += (s.empty() ? "" : ", ") + std::to_string(n);
            raise(PyExc_TypeError, std::string(name) + ": expected a contiguous CUDA tensor [" + s + "] of " + dtype_name(type));
        }
        here(o, name);
        return t->data_ptr();
    }
    void *dense_or_null(PyObject *o, at::ScalarType type, at::IntArrayRef shape, const char *name) const {
        return given(o) ? dense(o, type, shape, name) : nullptr;
    }
    at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) const { return at::empty(shape, at::TensorOptions().dtype(type).device(device)); }
    // Scratch of the call: the allocator gives it to nobody else before the work enqueued here is done
    at::Tensor scratch(int64_t bytes) const { return bytes > 0 ? empty({bytes}, at::kByte) : at::Tensor(); }

    template <typename F>
    void launch(F &&f) const {
        const c10::DeviceGuard guard(device);
        ::launch(f);
    }
};

bool truth(PyObject *o, bool otherwise) {
    if (!o) return otherwise;
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised{};
    return v != 0;
}
float real(PyObject *o, double otherwise) {
    if (!o) return (float)otherwise;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return (float)v;
}
void rows_of_sequences(int64_t M, int64_t B, int64_t L, const char *name) {
    if (B < 0 || L <= 0 || !is_product(M, B, L)) raise(PyExc_ValueError, std::string(name) + " must have B*L rows");
}
void *scratch_data(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
int64_t scratch_bytes(const at::Tensor &t) { return t.defined() ? t.numel() : 0; }
void not_the_same(const void *a, const void *b, const char *name) {
    if (a && a == b) raise(PyExc_ValueError, std::string(name) + ": not the buffer of state");
}

PyObject *wrap(const at::Tensor &t) {
    PyObject *o = THPVariable_Wrap(t);
    if (!o) throw Raised{};
    return o;
}
// The values as a tuple, None for a null pointer; the references stay with the callers' Owned
template <size_t N>
PyObject *tuple_of(PyObject *const (&items)[N]) {
    PyObject *t = PyTuple_New(N);
    if (!t) throw Raised{};
    for (size_t i = 0; i < N; i++) {
        PyObject *o = items[i] ? items[i] : Py_None;
        Py_INCREF(o);
        PyTuple_SET_ITEM(t, i, o);
    }
    return t;
}

struct ScanInputs {
    Matrix u, dt, b, c, z;
    const float *a, *d, *dt_bias;
    int64_t K, N;
    // u dt a b c d z dt_bias, from `at` on
    ScanInputs(const Operands &ops, Args at) : u(matrix(at[0], ops.dtype, "u")) {
        const int64_t M = u.rows;
        K = u.cols;
        ops.here(at[0], "u");
        const at::Tensor *t = tensor(at[2]);
        if (!t || t->dim() != 2) raise(PyExc_TypeError, "a: expected a contiguous CUDA tensor [K, N] of torch.float32");
        N = t->size(1);
        dt = ops.in(at[1], M, K, "dt");
        a = static_cast<const float *>(ops.dense(at[2], at::kFloat, {K, N}, "a"));
        b = ops.in(at[3], M, N, "b");
        c = ops.in(at[4], M, N, "c");
        d = ops.floats(at[5], K, "d", true);
        z = ops.optional(at[6], ops.dtype, M, K, "z");
        dt_bias = ops.floats(at[7], K, "dt_bias", true);
    }
};

PyObject *gated_scan(Args a) {  // u dt a b c d z dt_bias B L reverse state y state_out marks
    const Operands ops(a[0], "u");
    const ScanInputs in(ops, a);
    const int64_t B = integer(a[8]), L = integer(a[9]), K = in.K, N = in.N;
    rows_of_sequences(in.u.rows, B, L, "u");
    const bool reverse = truth(a[10], false);
    const float *state = floats(ops.dense_or_null(a[11], at::kFloat, {B, K, N}, "state"));
    Owned out(output(a[12], {in.u.rows, K}, ops.dtype, a[0]));
    const Matrix y = ops.out(out.o, ops.dtype, in.u.rows, K, "y");
    float *const state_out = static_cast<float *>(ops.dense_or_null(a[13], at::kFloat, {B, K, N}, "state_out"));
    not_the_same(state, state_out, "state_out");
    float *const marks = given(a[14]) ? static_cast<float *>(ops.dense(a[14], at::kFloat, {PTQ4VM_SCAN_MARKS(L), B, K, N}, "marks")) : nullptr;
    const at::Tensor ws = ops.scratch(entry.gated_scan_workspace(B, L, K, N));
    ops.launch([&](void *s) { return entry.gated_scan(ops.code, in.u.data, in.dt.data, in.a, in.b.data, in.c.data, in.d, in.z.data, in.dt_bias, state, y.data, state_out,
                               marks, scratch_data(ws), scratch_bytes(ws), reverse, B, L, K, N, in.u.ld, in.dt.ld, in.b.ld, in.c.ld, in.z.ld, y.ld, s); });
    return out.release();
}

PyObject *gated_scan_backward(Args a) {  // dy u dt a b c d z dt_bias marks B L reverse du ddt db dc dz
    const Operands ops(a[1], "u");
    const ScanInputs in(ops, a + 1);
    const int64_t B = integer(a[10]), L = integer(a[11]), M = in.u.rows, K = in.K, N = in.N;
    rows_of_sequences(M, B, L, "u");
    const Matrix dy = ops.in(a[0], M, K, "dy");
    const float *marks = floats(ops.dense(a[9], at::kFloat, {PTQ4VM_SCAN_MARKS(L), B, K, N}, "marks"));
    const bool reverse = truth(a[12], false);
    if (given(a[17]) && !in.z.data && !given(a[7])) raise(PyExc_ValueError, "dz: there is no z");
    Owned o_du(output(a[13], {M, K}, ops.dtype, a[1])), o_ddt(output(a[14], {M, K}, ops.dtype, a[1])), o_db(output(a[15], {M, N}, ops.dtype, a[1])),
        o_dc(output(a[16], {M, N}, ops.dtype, a[1])), o_dz(given(a[7]) ? output(a[17], {M, K}, ops.dtype, a[1]) : nullptr);
    const Matrix du = ops.out(o_du.o, ops.dtype, M, K, "du"), ddt = ops.out(o_ddt.o, ops.dtype, M, K, "ddt"), db = ops.out(o_db.o, ops.dtype, M, N, "db"),
                 dc = ops.out(o_dc.o, ops.dtype, M, N, "dc"), dz = o_dz.o ? ops.out(o_dz.o, ops.dtype, M, K, "dz") : Matrix{M, K, K, nullptr};
    const at::Tensor t_da = ops.empty({K, N}, at::kFloat), t_dd = given(a[6]) ? ops.empty({K}, at::kFloat) : at::Tensor(),
                     t_bias = given(a[8]) ? ops.empty({K}, at::kFloat) : at::Tensor();
    const at::Tensor ws = ops.scratch(entry.gated_scan_backward_workspace(B, L, K, N));
    const auto data = [](const at::Tensor &t) { return t.defined() ? static_cast<float *>(t.data_ptr()) : nullptr; };
    ops.launch([&](void *s) { return entry.gated_scan_backward(ops.code, dy.data, in.u.data, in.dt.data, in.a, in.b.data, in.c.data, in.d, in.z.data, in.dt_bias, marks, du.data,
                               ddt.data, data(t_da), db.data, dc.data, data(t_dd), dz.data, data(t_bias), scratch_data(ws), scratch_bytes(ws), reverse, B, L, K, N, dy.ld,
                               in.u.ld, in.dt.ld, in.b.ld, in.c.ld, in.z.ld, du.ld, ddt.ld, db.ld, dc.ld, dz.ld, s); });
    Owned da(wrap(t_da)), dd(t_dd.defined() ? wrap(t_dd) : nullptr), dbias(t_bias.defined() ? wrap(t_bias) : nullptr);
    return tuple_of({o_du.o, o_ddt.o, da.o, o_db.o, o_dc.o, dd.o, o_dz.o, dbias.o});
}

PyObject *gated_scan_step(Args a) {  // u dt a b c d z dt_bias state y state_out
    const Operands ops(a[0], "u");
    const ScanInputs in(ops, a);
    const int64_t B = in.u.rows, K = in.K, N = in.N;
    float *const state = static_cast<float *>(ops.dense(a[8], at::kFloat, {B, K, N}, "state"));
    Owned out(output(a[9], {B, K}, ops.dtype, a[0]));
    const Matrix y = ops.out(out.o, ops.dtype, B, K, "y");
    float *const state_out = given(a[10]) ? static_cast<float *>(ops.dense(a[10], at::kFloat, {B, K, N}, "state_out")) : state;
    ops.launch([&](void *s) { return entry.gated_scan_step(ops.code, in.u.data, in.dt.data, in.a, in.b.data, in.c.data, in.d, in.z.data, in.dt_bias, state, y.data, state_out, B,
                               K, N, in.u.ld, in.dt.ld, in.b.ld, in.c.ld, in.z.ld, y.ld, s); });
    return out.release();
}

struct ConvInputs {
    Matrix x;
    const float *w, *bias;
    int64_t K, W;
    ConvInputs(const Operands &ops, Args at) : x(matrix(at[0], ops.dtype, "x")) {  // x w bias, from `at` on
        K = x.cols;
        const at::Tensor *t = tensor(at[1]);
        if (!t || t->dim() != 2 || t->size(1) < 2 || t->size(1) > 4) raise(PyExc_TypeError, "w: expected a contiguous CUDA tensor [K, 2..4] of torch.float32");
        W = t->size(1);
        w = floats(ops.dense(at[1], at::kFloat, {K, W}, "w"));
        bias = ops.floats(at[2], K, "bias", true);
    }
};

PyObject *token_conv(Args a) {  // x w bias B L silu reverse state y state_out
    const Operands ops(a[0], "x");
    const ConvInputs in(ops, a);
    const int64_t B = integer(a[3]), L = integer(a[4]), K = in.K, W = in.W;
    rows_of_sequences(in.x.rows, B, L, "x");
    const bool silu = truth(a[5], true), reverse = truth(a[6], false);
    const void *state = ops.dense_or_null(a[7], ops.dtype, {B, W - 1, K}, "state");
    Owned out(output(a[8], {in.x.rows, K}, ops.dtype, a[0]));
    const Matrix y = ops.out(out.o, ops.dtype, in.x.rows, K, "y");
    void *const state_out = ops.dense_or_null(a[9], ops.dtype, {B, W - 1, K}, "state_out");
    not_the_same(state, state_out, "state_out");
    ops.launch([&](void *s) { return entry.token_conv(ops.code, in.x.data, in.w, in.bias, state, y.data, state_out, silu, reverse, B, L, K, W, in.x.ld, y.ld, s); });
    return out.release();
}

PyObject *token_conv_backward(Args a) {  // dy x w bias B L silu reverse state dx
    const Operands ops(a[1], "x");
    const ConvInputs in(ops, a + 1);
    const int64_t B = integer(a[4]), L = integer(a[5]), M = in.x.rows, K = in.K, W = in.W;
    rows_of_sequences(M, B, L, "x");
    const Matrix dy = ops.in(a[0], M, K, "dy");
    const bool silu = truth(a[6], true), reverse = truth(a[7], false);
    const void *state = ops.dense_or_null(a[8], ops.dtype, {B, W - 1, K}, "state");
    Owned o_dx(output(a[9], {M, K}, ops.dtype, a[1]));
    const Matrix dx = ops.out(o_dx.o, ops.dtype, M, K, "dx");
    const at::Tensor t_dw = ops.empty({K, W}, at::kFloat), t_db = given(a[3]) ? ops.empty({K}, at::kFloat) : at::Tensor();
    const at::Tensor ws = ops.scratch(entry.token_conv_backward_workspace(B, L, K, W));
    float *const dbias = t_db.defined() ? static_cast<float *>(t_db.data_ptr()) : nullptr;
    ops.launch([&](void *s) { return entry.token_conv_backward(ops.code, dy.data, in.x.data, in.w, in.bias, state, dx.data, static_cast<float *>(t_dw.data_ptr()), dbias,
                               scratch_data(ws), scratch_bytes(ws), silu, reverse, B, L, K, W, dy.ld, in.x.ld, dx.ld, s); });
    Owned o_dw(wrap(t_dw)), o_db(t_db.defined() ? wrap(t_db) : nullptr);
    return tuple_of({o_dx.o, o_dw.o, o_db.o});
}

PyObject *token_conv_step(Args a) {  // x w bias state silu y state_out
    const Operands ops(a[0], "x");
    const ConvInputs in(ops, a);
    const int64_t B = in.x.rows, K = in.K, W = in.W;
    void *const state = ops.dense(a[3], ops.dtype, {B, W - 1, K}, "state");
    const bool silu = truth(a[4], true);
    Owned out(output(a[5], {B, K}, ops.dtype, a[0]));
    const Matrix y = ops.out(out.o, ops.dtype, B, K, "y");
    void *const state_out = given(a[6]) ? ops.dense(a[6], ops.dtype, {B, W - 1, K}, "state_out") : state;
    ops.launch([&](void *s) { return entry.token_conv_step(ops.code, in.x.data, in.w, in.bias, state, y.data, state_out, silu, B, K, W, in.x.ld, y.ld, s); });
    return out.release();
}

// The residual stream's type: that of the first of these that is given
at::ScalarType stream_type(const Operands &ops, PyObject *o, PyObject *other, const char *name) {
    const at::Tensor *t = given(o) ? tensor(o) : given(other) ? tensor(other) : nullptr;
    if (!given(o) && !given(other)) return ops.dtype;
    if (!t || (t->scalar_type() != ops.dtype && t->scalar_type() != at::kFloat))
        raise(PyExc_TypeError, std::string(name) + ": expected a 2-D CUDA tensor of " + dtype_name(ops.dtype) + " or torch.float32");
    return t->scalar_type();
}
struct Gate {
    const float *data = nullptr;
    int64_t rows = 0;
    Gate(const Operands &ops, PyObject *o, int64_t M, int64_t K) {
        if (!given(o)) return;
        const at::Tensor *t = tensor(o);
        if (!t || t->dim() != 2) raise(PyExc_TypeError, "gate: expected a contiguous CUDA tensor [G, K] of torch.float32");
        rows = t->size(0);
        data = floats(ops.dense(o, at::kFloat, {rows, K}, "gate"));
        if (rows <= 0 || M % rows != 0) raise(PyExc_ValueError, "gate: its rows must divide those of h");
    }
};

PyObject *residual_norm(Args a) {  // h residual w gate w_post scale eps y residual_out
    const Operands ops(a[0], "h");
    const Matrix h = matrix(a[0], ops.dtype, "h");
    const int64_t M = h.rows, K = h.cols;
    const at::ScalarType type = stream_type(ops, a[1], a[8], given(a[1]) ? "residual" : "residual_out");
    const Matrix residual = ops.optional(a[1], type, M, K, "residual");
    const float *w = ops.floats(a[2], K, "w"), *w_post = ops.floats(a[4], K, "w_post", true);
    const Gate gate(ops, a[3], M, K);
    const float scale = real(a[5], 1.0), eps = real(a[6], 1e-5);
    Owned o_y(output(a[7], {M, K}, ops.dtype, a[0])), o_r(output(a[8], {M, K}, type, a[0]));
    const Matrix y = ops.out(o_y.o, ops.dtype, M, K, "y"), r = ops.out(o_r.o, type, M, K, "residual_out");
    ops.launch([&](void *s) { return entry.residual_norm(ops.code, Operands::code_of(type), h.data, residual.data, w, gate.data, w_post, y.data, r.data, scale, eps, M, K, gate.rows,
                               h.ld, residual.ld, y.ld, r.ld, s); });
    return tuple_of({o_y.o, o_r.o});
}

PyObject *residual_norm_backward(Args a) {  // dy dr h r w gate w_post scale eps first dh dresidual
    const Operands ops(a[2], "h");
    const Matrix h = matrix(a[2], ops.dtype, "h");
    const int64_t M = h.rows, K = h.cols;
    const Matrix dy = ops.in(a[0], M, K, "dy");
    const at::ScalarType type = stream_type(ops, a[3], nullptr, "r");
    const Matrix r = ops.in(a[3], type, M, K, "r"), dr = ops.optional(a[1], type, M, K, "dr");
    const float *w = ops.floats(a[4], K, "w"), *w_post = ops.floats(a[6], K, "w_post", true);
    const Gate gate(ops, a[5], M, K);
    const float scale = real(a[7], 1.0), eps = real(a[8], 1e-5);
    const bool first = truth(a[9], false);
    if (first && given(a[11])) raise(PyExc_ValueError, "dresidual: there is no residual");
    Owned o_dh(output(a[10], {M, K}, ops.dtype, a[2])), o_dres(first ? nullptr : output(a[11], {M, K}, type, a[2]));
    const Matrix dh = ops.out(o_dh.o, ops.dtype, M, K, "dh"), dres = first ? Matrix{M, K, K, nullptr} : ops.out(o_dres.o, type, M, K, "dresidual");
    const at::Tensor t_dw = ops.empty({K}, at::kFloat), t_dgate = gate.data || given(a[5]) ? ops.empty({gate.rows, K}, at::kFloat) : at::Tensor(),
                     t_dpost = w_post ? ops.empty({K}, at::kFloat) : at::Tensor();
    const at::Tensor ws = ops.scratch(entry.residual_norm_backward_workspace(M, K, gate.rows));
    const auto data = [](const at::Tensor &t) { return t.defined() ? static_cast<float *>(t.data_ptr()) : nullptr; };
    ops.launch([&](void *s) { return entry.residual_norm_backward(ops.code, Operands::code_of(type), dy.data, dr.data, h.data, r.data, w, gate.data, w_post, dh.data, dres.data,
                               data(t_dw), data(t_dgate), data(t_dpost), scratch_data(ws), scratch_bytes(ws), scale, eps, M, K, gate.rows, dy.ld, dr.ld, h.ld, r.ld, dh.ld,
                               dres.ld, s); });
    Owned dw(wrap(t_dw)), dgate(t_dgate.defined() ? wrap(t_dgate) : nullptr), dpost(t_dpost.defined() ? wrap(t_dpost) : nullptr);
    return tuple_of({o_dh.o, o_dres.o, dw.o, dgate.o, dpost.o});
}

// ---------------------------------------------------------------------------------- Python signatures
constexpr int kMaxParams = 18;

struct Signature {
    const char *function;
    int required, total;
    const char *names[kMaxParams];
    PyObject *interned[kMaxParams];
};

// Python's calling convention: positional arguments, then keywords; missing optional ones stay null.
void parse(const Signature &sig, Args args, Py_ssize_t nargs, PyObject *kwnames, PyObject **out) {
    if (nargs > sig.total)
        raise(PyExc_TypeError, std::string(sig.function) + "() takes at most " + std::to_string(sig.total) + " arguments (" + std::to_string(nargs) + " given)");
    for (Py_ssize_t i = 0; i < nargs; i++) out[i] = args[i];
    for (int i = (int)nargs; i < sig.total; i++) out[i] = nullptr;
    const Py_ssize_t n_kw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < n_kw; k++) {
        PyObject *name = PyTuple_GET_ITEM(kwnames, k);
        int at = -1;
        for (int i = 0; i < sig.total && at < 0; i++)
            if (sig.interned[i] == name) at = i;
        for (int i = 0; i < sig.total && at < 0; i++)
            if (PyUnicode_CompareWithASCIIString(name, sig.names[i]) == 0) at = i;
        if (at < 0) {
            PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", sig.function, name);
            throw Raised{};
        }
        if (out[at]) {
            PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%U'", sig.function, name);
            throw Raised{};
        }
        out[at] = args[nargs + k];
    }
    for (int i = 0; i < sig.required; i++)
        if (!out[i]) raise(PyExc_TypeError, std::string(sig.function) + "() missing required argument: '" + sig.names[i] + "'");
}

// Inside a catch block: the exception as torch raises it (torch.OutOfMemoryError).  Apart from the call itself, because
// torch's macros set up a warning handler on the way in, 0.2 us a call.
PyObject *raise_as_torch() {
    HANDLE_TH_ERRORS
    throw;
    END_HANDLE_TH_ERRORS
}

template <PyObject *(*CALL)(Args), Signature *SIG>
PyObject *call(PyObject *, Args args, Py_ssize_t nargs, PyObject *kwnames) {
    try {
        PyObject *a[kMaxParams];
        parse(*SIG, args, nargs, kwnames, a);
        need_library();
        return CALL(a);
    } catch (const Raised &) {
        return nullptr;
    } catch (...) {  // an output that could not be allocated
        return raise_as_torch();
    }
}

#define SIG(name, required, total, ...) Signature sig_##name = {#name, required, total, {__VA_ARGS__}, {}};
SIG(quantize_pts, 5, 6, "x", "inv_m", "s_tok", "B", "L", "xq")
SIG(quantize_dynamic, 2, 4, "x", "inv_m", "xq", "s_row")
SIG(quantize_pts_offset, 6, 7, "x", "inv_m", "s_tok", "z_tok", "B", "L", "xq")
SIG(quantize_pts_a4, 5, 6, "x", "inv_m", "s_tok", "B", "L", "xq4")
SIG(quantize_pts_a4_e2m3, 5, 6, "x", "inv_m", "s_tok", "B", "L", "xq6")
SIG(w8a8_linear, 7, 9, "xq", "wq", "s_tok", "s_w", "bias", "B", "L", "y", "acc_out")
SIG(w8a8_linear_offset, 9, 11, "xq", "wq", "s_tok", "z_tok", "rowsum", "s_w", "bias", "B", "L", "y", "acc_out")
SIG(w4a4_linear, 7, 9, "xq4", "wq4", "s_tok", "s_w", "bias", "B", "L", "y", "acc_out")
SIG(w4a4_linear_e2m3, 8, 10, "xq6", "wq6", "s_tok", "s_w", "bias", "B", "L", "K", "y", "acc_out")
SIG(w8a8_linear_fused, 8, 11, "x", "inv_m", "s_tok", "wq", "s_w", "bias", "B", "L", "y", "acc_out", "xq_out")
SIG(w8a8_linear_offset_fused, 10, 13, "x", "inv_m", "s_tok", "z_tok", "wq", "rowsum", "s_w", "bias", "B", "L", "y", "acc_out", "xq_out")
SIG(w4a4_linear_fused, 8, 11, "x", "inv_m", "s_tok", "wq4", "s_w", "bias", "B", "L", "y", "acc_out", "xq_out")
SIG(f16_linear, 3, 4, "x", "w", "bias", "y")
SIG(gated_scan, 10, 15, "u", "dt", "a", "b", "c", "d", "z", "dt_bias", "B", "L", "reverse", "state", "y", "state_out", "marks")
SIG(gated_scan_backward, 12, 18, "dy", "u", "dt", "a", "b", "c", "d", "z", "dt_bias", "marks", "B", "L", "reverse", "du", "ddt", "db", "dc", "dz")
SIG(gated_scan_step, 9, 11, "u", "dt", "a", "b", "c", "d", "z", "dt_bias", "state", "y", "state_out")
SIG(token_conv, 5, 10, "x", "w", "bias", "B", "L", "silu", "reverse", "state", "y", "state_out")
SIG(token_conv_backward, 6, 10, "dy", "x", "w", "bias", "B", "L", "silu", "reverse", "state", "dx")
SIG(token_conv_step, 4, 7, "x", "w", "bias", "state", "silu", "y", "state_out")
SIG(residual_norm, 3, 9, "h", "residual", "w", "gate", "w_post", "scale", "eps", "y", "residual_out")
SIG(residual_norm_backward, 5, 12, "dy", "dr", "h", "r", "w", "gate", "w_post", "scale", "eps", "first", "dh", "dresidual")
#undef SIG

// bind({name: address of ptq4vm_<name>}): the entry points of the loaded library
PyObject *bind(PyObject *, PyObject *table) {
#define X(name)                                                                                        \
    {                                                                                                  \
        PyObject *v = PyDict_GetItemString(table, #name);                                              \
        if (!v) return PyErr_Format(PyExc_KeyError, "ptq4vm_%s", #name);                               \
        entry.name = reinterpret_cast<decltype(&ptq4vm_##name)>(PyLong_AsVoidPtr(v));                  \
        if (!entry.name) return PyErr_Format(PyExc_ValueError, "ptq4vm_%s: no address", #name);        \
    }
    PTQ4VM_HOT_ENTRIES(X)
#undef X
    bound = true;
    Py_RETURN_NONE;
}

// setup(load_library, raise_status): the two Python callbacks
PyObject *setup(PyObject *, PyObject *args) {
    PyObject *load, *status;
    if (!PyArg_ParseTuple(args, "OO", &load, &status)) return nullptr;
    Py_INCREF(load);
    Py_INCREF(status);
    Py_XSETREF(load_library, load);
    Py_XSETREF(raise_status, status);
    Py_RETURN_NONE;
}

#define FAST(name, doc) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call<name, &sig_##name>)), METH_FASTCALL | METH_KEYWORDS, doc}
PyMethodDef methods[] = {
    FAST(quantize_pts, "quantize_pts(x, inv_m, s_tok, B, L, xq=None)\n--\n\nptq4vm_quantize_pts: xq int8 [B*L, K]."),
    FAST(quantize_dynamic, "quantize_dynamic(x, inv_m, xq=None, s_row=None)\n--\n\nptq4vm_quantize_dynamic: (xq int8 [M, K], s_row f32 [M])."),
    FAST(quantize_pts_offset, "quantize_pts_offset(x, inv_m, s_tok, z_tok, B, L, xq=None)\n--\n\n"
                              "ptq4vm_quantize_pts_offset: xq int8 [B*L, K] with the per-token zero offset z_tok (int32 [L])."),
    FAST(quantize_pts_a4, "quantize_pts_a4(x, inv_m, s_tok, B, L, xq4=None)\n--\n\n"
                          "ptq4vm_quantize_pts_a4: xq4 uint8 [B*L, K/2], two 4-bit codes per byte."),
    FAST(quantize_pts_a4_e2m3, "quantize_pts_a4_e2m3(x, inv_m, s_tok, B, L, xq6=None)\n--\n\n"
                               "ptq4vm_quantize_pts_a4_e2m3: xq6 uint8 [e2m3_blocks(K), B*L, 96], 4-bit codes as E2M3 patterns, block-major."),
    FAST(w8a8_linear, "w8a8_linear(xq, wq, s_tok, s_w, bias, B, L, y=None, acc_out=None)\n--\n\n"
                      "ptq4vm_w8a8_linear: y fp16 [B*L, N]; acc_out (int32 [B*L, N], dense) is filled if given."),
    FAST(w8a8_linear_offset, "w8a8_linear_offset(xq, wq, s_tok, z_tok, rowsum, s_w, bias, B, L, y=None, acc_out=None)\n--\n\n"
                             "ptq4vm_w8a8_linear_offset: y fp16 [B*L, N] with the zero-offset correction in the epilogue."),
    FAST(w4a4_linear, "w4a4_linear(xq4, wq4, s_tok, s_w, bias, B, L, y=None, acc_out=None)\n--\n\n"
                      "ptq4vm_w4a4_linear: y fp16 [B*L, N] from packed 4-bit operands."),
    FAST(w4a4_linear_e2m3, "w4a4_linear_e2m3(xq6, wq6, s_tok, s_w, bias, B, L, K, y=None, acc_out=None)\n--\n\n"
                           "ptq4vm_w4a4_linear_e2m3: y fp16 [B*L, N] from operands in the block-major E2M3 container (K codes per row)."),
    FAST(w8a8_linear_fused, "w8a8_linear_fused(x, inv_m, s_tok, wq, s_w, bias, B, L, y=None, acc_out=None, xq_out=None)\n--\n\n"
                            "ptq4vm_w8a8_linear_fused: y fp16 [B*L, N] from fp16 activations; acc_out / xq_out are filled if given."),
    FAST(w8a8_linear_offset_fused,
         "w8a8_linear_offset_fused(x, inv_m, s_tok, z_tok, wq, rowsum, s_w, bias, B, L, y=None, acc_out=None, xq_out=None)\n--\n\n"
         "ptq4vm_w8a8_linear_offset_fused: y fp16 [B*L, N] from fp16 activations, per-token steps and zero offsets;\n"
         "acc_out (raw accumulators) / xq_out (codes with the offset in them) are filled if given."),
    FAST(w4a4_linear_fused, "w4a4_linear_fused(x, inv_m, s_tok, wq4, s_w, bias, B, L, y=None, acc_out=None, xq_out=None)\n--\n\n"
                            "ptq4vm_w4a4_linear_fused: y fp16 [B*L, N] from fp16 activations and a packed 4-bit weight [N, K/2];\n"
                            "acc_out / xq_out (int8, one 4-bit code per byte) are filled if given."),
    FAST(f16_linear, "f16_linear(x, w, bias, y=None)\n--\n\nptq4vm_f16_linear: y fp16 [M, N]."),
    FAST(gated_scan, "gated_scan(u, dt, a, b, c, d, z, dt_bias, B, L, reverse=False, state=None, y=None, state_out=None, marks=None)\n--\n\n"
                     "ptq4vm_gated_scan: y [B*L, K] of u's type (fp16, bfloat16, fp32); state_out (f32 [B, K, N], not state itself) and marks\n"
                     "(f32 [scan_marks(L), B, K, N], for the backward pass) are filled if given.  Records nothing for autograd: gradients come from\n"
                     "gated_scan_backward, called with the same arguments."),
    FAST(gated_scan_backward, "gated_scan_backward(dy, u, dt, a, b, c, d, z, dt_bias, marks, B, L, reverse=False, du=None, ddt=None, db=None, dc=None, dz=None)\n--\n\n"
                              "ptq4vm_gated_scan_backward: (du, ddt, da, db, dc, dd, dz, ddt_bias); None for the gradient of an input that is None."),
    FAST(gated_scan_step, "gated_scan_step(u, dt, a, b, c, d, z, dt_bias, state, y=None, state_out=None)\n--\n\n"
                          "ptq4vm_gated_scan_step: y [B, K] for one token of each sequence; state (f32 [B, K, N]) advances in place unless state_out is given."),
    FAST(token_conv, "token_conv(x, w, bias, B, L, silu=True, reverse=False, state=None, y=None, state_out=None)\n--\n\n"
                     "ptq4vm_token_conv: y [B*L, K] of x's type, apart from x; state_out ([B, W - 1, K] of x's type, not state itself) is filled if given.\n"
                     "Records nothing for autograd: gradients come from token_conv_backward."),
    FAST(token_conv_backward, "token_conv_backward(dy, x, w, bias, B, L, silu=True, reverse=False, state=None, dx=None)\n--\n\n"
                              "ptq4vm_token_conv_backward: (dx, dw, dbias); dx is apart from x and dy, dbias None without a bias."),
    FAST(token_conv_step, "token_conv_step(x, w, bias, state, silu=True, y=None, state_out=None)\n--\n\n"
                          "ptq4vm_token_conv_step: y [B, K] for one token of each sequence; state ([B, W - 1, K]) advances in place unless state_out is given."),
    FAST(residual_norm, "residual_norm(h, residual, w, gate=None, w_post=None, scale=1.0, eps=1e-5, y=None, residual_out=None)\n--\n\n"
                        "ptq4vm_residual_norm: (y, residual_out); residual_out has residual's type, h's where residual is None and none is given.\n"
                        "Records nothing for autograd: gradients come from residual_norm_backward."),
    FAST(residual_norm_backward, "residual_norm_backward(dy, dr, h, r, w, gate=None, w_post=None, scale=1.0, eps=1e-5, first=False, dh=None, dresidual=None)\n--\n\n"
                                 "ptq4vm_residual_norm_backward, r the forward pass's residual_out and dr its gradient or None: (dh, dresidual, dw, dgate,\n"
                                 "dw_post); dresidual is None with first=True (no residual), dgate and dw_post without gate and w_post."),
    {"bind", bind, METH_O, "bind(table)\n--\n\nAddresses of the library's entry points by name, without the ptq4vm_ prefix."},
    {"setup", setup, METH_VARARGS, "setup(load_library, raise_status)\n--\n\nCallbacks: load the library and bind(); raise for a status."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Launches of libptq4vm.so as Python callables.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    for (Signature *s : {&sig_quantize_pts, &sig_quantize_dynamic, &sig_quantize_pts_offset, &sig_quantize_pts_a4, &sig_quantize_pts_a4_e2m3,
                         &sig_w8a8_linear, &sig_w8a8_linear_offset, &sig_w4a4_linear, &sig_w4a4_linear_e2m3, &sig_w8a8_linear_fused,
                         &sig_w8a8_linear_offset_fused, &sig_w4a4_linear_fused, &sig_f16_linear, &sig_gated_scan, &sig_gated_scan_backward,
                         &sig_gated_scan_step, &sig_token_conv, &sig_token_conv_backward, &sig_token_conv_step, &sig_residual_norm, &sig_residual_norm_backward})
        for (int i = 0; i < s->total; i++) s->interned[i] = PyUnicode_InternFromString(s->names[i]);
    return PyModule_Create(&module);
}
