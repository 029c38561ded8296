// Argument marshalling of the enqueuing entry points (include/xnor.h) for Python: device tensors to addresses, one C call
// each.  A layer's launch takes the GPU 2 to 5 us at the smallest sizes, less than the same checks and conversions
// cost through ctypes (5.3 us of host time per call, HIP's launch of about 2 us included; 3.5 us here): one 64 x 14 x 14
// block, two calls, 11.6 -> 8.5 us; one row of a 9216 -> 4096 layer 11.2 -> 7.6 us.
//
// Checks of a tensor argument: NULL or a dense device tensor of the stated type, as the callers of xnor.py have always
// been told; sizes are the caller's, as in the C ABI.  The library's entry points are looked up in the file that xnor.py
// names (bind), so that another build of it can be called.
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/autograd/python_variable.h>

#include <dlfcn.h>

#include "xnor.h"
#include "xnor_lowbit.h"

namespace {

// The Python error that is already set (thrown so that every exit path of a call is the same).
struct PythonError {};

PyObject *g_raise = nullptr;            // xnor.py's error for a non-zero status: raise(name, status)
PyObject *g_desc = nullptr;             // xnor.py's descriptor class
PyObject *g_current_device = nullptr, *g_raw_stream = nullptr;      // torch's, for calls without a stream

[[noreturn]] void fail(PyObject *type, const char *message)
{
    PyErr_SetString(type, message);
    throw PythonError{};
}

void *tensor(PyObject *o, c10::ScalarType type)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor or None");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) fail(PyExc_ValueError, "libxnor takes device tensors");
    if (!t.is_contiguous()) fail(PyExc_ValueError, "libxnor takes densely packed tensors");
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_ValueError, "expected %s, got %s", c10::toString(type), c10::toString(t.scalar_type()));
        throw PythonError{};
    }
    return t.data_ptr();
}
float *f32(PyObject *o) { return static_cast<float *>(tensor(o, c10::ScalarType::Float)); }
uint32_t *u32(PyObject *o) { return static_cast<uint32_t *>(tensor(o, c10::ScalarType::Int)); }
int32_t *i32(PyObject *o) { return static_cast<int32_t *>(tensor(o, c10::ScalarType::Int)); }
void *u8(PyObject *o) { return tensor(o, c10::ScalarType::Byte); }

int num(PyObject *o)
{
    const unsigned long v = PyLong_AsUnsignedLongMask(o);           // (C's conversion to int, as ctypes has it)
    if (v == (unsigned long)-1 && PyErr_Occurred()) throw PythonError{};
    return (int)v;
}
int64_t area(PyObject *n, PyObject *m) { return (int64_t)num(n) * num(m); }

double real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
    return v;
}

// Arguments of the calls of xnor_lowbit.h.  Their tensors are looked at more closely, since a row too few is a read out of range: each has to
// hold what the sizes say.
c10::ScalarType scalar_type(int type)
{
    return type == XNOR_F32 ? c10::ScalarType::Float : type == XNOR_BF16 ? c10::ScalarType::BFloat16 : c10::ScalarType::Half;
}
// the xnor_dtype of a real tensor
int dtype(PyObject *o)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor");
    switch (THPVariable_Unpack(o).scalar_type()) {
    case c10::ScalarType::Float: return XNOR_F32;
    case c10::ScalarType::BFloat16: return XNOR_BF16;
    case c10::ScalarType::Half: return XNOR_F16;
    default: fail(PyExc_ValueError, "expected float32, bfloat16 or float16");
    }
}
int token_bytes(PyObject *o)
{
    if (o == Py_None) return 4;
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor or None");
    switch (THPVariable_Unpack(o).scalar_type()) {
    case c10::ScalarType::Int: return 4;
    case c10::ScalarType::Long: return 8;
    default: fail(PyExc_ValueError, "expected int32 or int64 tokens");
    }
}
void *dense(PyObject *o, c10::ScalarType type, int64_t count)
{
    void *p = tensor(o, type);
    if (o != Py_None && THPVariable_Unpack(o).numel() < count) fail(PyExc_ValueError, "a tensor holds less than the sizes say");
    return p;
}
float *dense_f32(PyObject *o, int64_t count) { return static_cast<float *>(dense(o, c10::ScalarType::Float, count)); }
void *tokens(PyObject *o, int64_t count) { return dense(o, token_bytes(o) == 8 ? c10::ScalarType::Long : c10::ScalarType::Int, count); }
template <class T> T *dense_of(PyObject *o, c10::ScalarType type, int64_t count) { return static_cast<T *>(dense(o, type, count)); }

// Rows of `cols` neighbours: a matrix whose rows may lie apart, or any dense tensor of that many elements.
bool lie_apart(const at::Tensor &t, int64_t rows, int64_t cols)
{
    return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && rows > 1 && t.stride(0) > cols && (cols == 1 || t.stride(1) == 1);
}
void *rows(PyObject *o, int type, int64_t n, int64_t cols)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor or None");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.is_cuda() && t.scalar_type() == scalar_type(type) && lie_apart(t, n, cols)) return t.data_ptr();
    return dense(o, scalar_type(type), n * cols);
}
int64_t stride(PyObject *o, int64_t n, int64_t cols)
{
    if (o == Py_None) return cols;
    const at::Tensor &t = THPVariable_Unpack(o);
    return lie_apart(t, n, cols) ? t.stride(0) : cols;
}
int64_t groups(int64_t cols, int64_t group) { return group > 0 ? (cols + group - 1) / group : 1; }

// Sizes that the library states, for the checks of images and workspaces.
#define XNOR_QUERIES(X)                                                                               \
    X(xnor_rmsnorm_backward_workspace_bytes) X(xnor_w4_wimg_bytes) X(xnor_w4_linear_workspace_bytes) \
    X(xnor_logprobs_workspace_bytes) X(xnor_w8_linear_workspace_bytes)                               \
    X(xnor_q8_weight_gradient_workspace_bytes) X(xnor_sample_workspace_bytes)
#define XNOR_QUERY_POINTER(NAME) decltype(&::NAME) p_##NAME = nullptr;
XNOR_QUERIES(XNOR_QUERY_POINTER)
void *bytes(PyObject *o, size_t count) { return dense(o, c10::ScalarType::Byte, (int64_t)count); }

// The device of a stream object, -1 where it does not say (a handle by itself).
int device_of(PyObject *stream)
{
    PyObject *device = PyObject_GetAttrString(stream, "device");
    if (!device) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) throw PythonError{};
        PyErr_Clear();
        return -1;
    }
    const int index = THPDevice_Check(device) ? (int)reinterpret_cast<THPDevice *>(device)->device.index() : -1;
    Py_DECREF(device);
    return index;
}
// The tensors among a call's arguments have to be on one device, that of the stream (the last argument) or, where none is given, the current one: a kernel would
// read another's memory, or run on a device that does not hold its tensors.  Returns `value`, so that a call's last number can stand for the check.
int on_one_device(PyObject *const *a, int n, int value)
{
    int device = a[n - 1] == Py_None ? (int)c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index() : device_of(a[n - 1]);
    for (int i = 0; i < n - 1; ++i) {
        if (!THPVariable_Check(a[i])) continue;
        const int here = (int)THPVariable_Unpack(a[i]).get_device();
        if (device >= 0 && here != device) fail(PyExc_ValueError, "the tensors of a call have to be on the device that it runs on");
        device = here;
    }
    return value;
}
int64_t wide(PyObject *cols, PyObject *gated) { return (int64_t)num(cols) << (num(gated) & 1); }

// A descriptor (xnor.py's ctypes structure, nothing else that holds as many bytes) through the buffer protocol; held for the
// duration of the call.
struct Desc {
    Py_buffer view{};
    explicit Desc(PyObject *o)
    {
        const int is = PyObject_IsInstance(o, g_desc);
        if (is < 0) throw PythonError{};
        if (!is) fail(PyExc_TypeError, "expected a convolution descriptor");
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw PythonError{};
        if (view.len != (Py_ssize_t)sizeof(xnor_conv_desc)) {
            PyBuffer_Release(&view);
            fail(PyExc_TypeError, "expected a convolution descriptor");
        }
    }
    ~Desc() { PyBuffer_Release(&view); }
    Desc(const Desc &) = delete;
    operator const xnor_conv_desc *() const { return static_cast<const xnor_conv_desc *>(view.buf); }
};

void *stream(PyObject *o)
{
    PyObject *handle;
    if (o != Py_None) {
        handle = PyObject_GetAttrString(o, "cuda_stream");
    } else {
        PyObject *device = PyObject_CallNoArgs(g_current_device);
        if (!device) throw PythonError{};
        handle = PyObject_CallOneArg(g_raw_stream, device);
        Py_DECREF(device);
    }
    if (!handle) throw PythonError{};
    void *s = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!s && PyErr_Occurred()) throw PythonError{};
    return s;
}

// Every entry point: its address in the bound library and the conversion of its arguments, in the C order with the stream
// last.
#define XNOR_CALLS(X)                                                                                                     \
    X(xnor_binarize_pack, 9, f32(a[0]), f32(a[1]), f32(a[2]), u32(a[3]), num(a[4]), num(a[5]), num(a[6]), num(a[7]))      \
    X(xnor_compute_K, 7, f32(a[0]), f32(a[1]), f32(a[2]), f32(a[3]), f32(a[4]), Desc(a[5]))                               \
    X(xnor_binactiv, 8, f32(a[0]), f32(a[1]), f32(a[2]), u32(a[3]), f32(a[4]), f32(a[5]), Desc(a[6]))                     \
    X(xnor_binactiv_streamed, 8, f32(a[0]), f32(a[1]), f32(a[2]), u32(a[3]), f32(a[4]), f32(a[5]), Desc(a[6]))            \
    X(xnor_pool_binactiv, 17, f32(a[0]), f32(a[1]), f32(a[2]), u32(a[3]), f32(a[4]), num(a[5]), num(a[6]), num(a[7]),     \
      num(a[8]), num(a[9]), num(a[10]), num(a[11]), num(a[12]), num(a[13]), num(a[14]), num(a[15]))                       \
    X(xnor_bwn_split, 7, f32(a[0]), u8(a[1]), num(a[2]), num(a[3]), num(a[4]), num(a[5]))                                 \
    X(xnor_bwn_pack_weights, 8, f32(a[0]), f32(a[1]), u8(a[2]), num(a[3]), num(a[4]), num(a[5]), num(a[6]))               \
    X(xnor_bwn_conv2d, 6, u8(a[0]), u8(a[1]), f32(a[2]), f32(a[3]), Desc(a[4]))                                           \
    X(xnor_bingrad_pack_weights, 9, f32(a[0]), u32(a[1]), f32(a[2]), u8(a[3]), num(a[4]), num(a[5]), num(a[6]), num(a[7]))\
    X(xnor_bingrad_binarize, 7, f32(a[0]), f32(a[1]), f32(a[2]), u32(a[3]), f32(a[4]), Desc(a[5]))                        \
    X(xnor_bingrad_conv2d, 11, u32(a[0]), u32(a[1]), u8(a[2]), f32(a[3]), f32(a[4]), f32(a[5]), f32(a[6]), i32(a[7]),     \
      Desc(a[8]), num(a[9]))                                                                                              \
    X(xnor_kbit_pack_input, 8, f32(a[0]), u8(a[1]), num(a[2]), num(a[3]), num(a[4]), num(a[5]), num(a[6]))                \
    X(xnor_kbit_pack_weights, 10, f32(a[0]), f32(a[1]), u8(a[2]), num(a[3]), num(a[4]), num(a[5]), num(a[6]), num(a[7]),  \
      num(a[8]))                                                                                                          \
    X(xnor_kbit_conv2d, 9, u8(a[0]), u8(a[1]), f32(a[2]), f32(a[3]), i32(a[4]), Desc(a[5]), num(a[6]), num(a[7]))         \
    X(xnor_pack_weights, 9, f32(a[0]), u32(a[1]), f32(a[2]), u8(a[3]), num(a[4]), num(a[5]), num(a[6]), num(a[7]))        \
    X(xnor_conv2d, 11, u32(a[0]), u32(a[1]), u8(a[2]), f32(a[3]), f32(a[4]), f32(a[5]), f32(a[6]), i32(a[7]), Desc(a[8]), \
      num(a[9]))                                                                                                          \
    X(xnor_conv2d_pool, 13, u32(a[0]), u8(a[1]), f32(a[2]), f32(a[3]), f32(a[4]), f32(a[5]), Desc(a[6]), num(a[7]),       \
      num(a[8]), num(a[9]), num(a[10]), num(a[11]))                                                                       \
    X(xnor_linear, 12, u32(a[0]), u32(a[1]), u8(a[2]), f32(a[3]), f32(a[4]), f32(a[5]), i32(a[6]), num(a[7]), num(a[8]),  \
      num(a[9]), num(a[10]))                                                                                              \
    X(xnor_conv2d_binactiv, 15, u32(a[0]), u32(a[1]), u8(a[2]), f32(a[3]), f32(a[4]), f32(a[5]), f32(a[6]), f32(a[7]),    \
      u32(a[8]), f32(a[9]), f32(a[10]), u8(a[11]), Desc(a[12]), num(a[13]))                                               \
    X(xnor_conv2d_binactiv_noalloc, 14, u32(a[0]), u32(a[1]), u8(a[2]), f32(a[3]), f32(a[4]), f32(a[5]), f32(a[6]),       \
      f32(a[7]), u32(a[8]), f32(a[9]), f32(a[10]), Desc(a[11]), num(a[12]))                                               \
    X(xnor_rmsnorm_q8, 13, rows(a[0], dtype(a[0]), num(a[8]), num(a[9])), stride(a[0], num(a[8]), num(a[9])),             \
      rows(a[1], dtype(a[0]), num(a[8]), num(a[9])), stride(a[1], num(a[8]), num(a[9])), dense_f32(a[2], num(a[9])),      \
      dense(a[3], scalar_type(dtype(a[0])), area(a[8], a[9])),                                                            \
      dense_of<int8_t>(a[4], c10::ScalarType::Char, area(a[8], a[9])),                                                    \
      dense_f32(a[5], num(a[8]) * groups(num(a[9]), num(a[10]))), dense(a[6], scalar_type(dtype(a[0])), area(a[8], a[9])),\
      dense_f32(a[7], num(a[8])), num(a[8]), num(a[9]), num(a[10]), dtype(a[0]), (float)real(a[11]))                      \
    X(xnor_rmsnorm_backward, 11, rows(a[0], dtype(a[0]), num(a[8]), num(a[9])), stride(a[0], num(a[8]), num(a[9])),       \
      dense_f32(a[1], num(a[8])), dense_f32(a[2], num(a[9])), rows(a[3], dtype(a[0]), num(a[8]), num(a[9])),              \
      stride(a[3], num(a[8]), num(a[9])), rows(a[4], dtype(a[0]), num(a[8]), num(a[9])),                                  \
      stride(a[4], num(a[8]), num(a[9])), dense(a[5], scalar_type(dtype(a[0])), area(a[8], a[9])),                        \
      dense_f32(a[6], num(a[9])), bytes(a[7], p_xnor_rmsnorm_backward_workspace_bytes(num(a[8]), num(a[9]))), num(a[8]),  \
      num(a[9]), dtype(a[0]))                                                                                             \
    X(xnor_w4_quantize, 8, rows(a[0], dtype(a[0]), num(a[4]), num(a[5])), stride(a[0], num(a[4]), num(a[5])),             \
      dense_of<uint8_t>(a[1], c10::ScalarType::Byte, num(a[4]) * groups(num(a[5]), 32) * 16),                             \
      dense_f32(a[2], num(a[4]) * groups(num(a[5]), num(a[6]))),                                                          \
      dense_of<uint8_t>(a[3], c10::ScalarType::Byte, num(a[4]) * groups(num(a[5]), num(a[6]))), num(a[4]), num(a[5]),     \
      num(a[6]), dtype(a[0]))                                                                                             \
    X(xnor_w4_pack, 8, dense_of<uint8_t>(a[0], c10::ScalarType::Byte, num(a[4]) * groups(num(a[5]), 32) * 16),            \
      dense_f32(a[1], num(a[4]) * groups(num(a[5]), num(a[6]))),                                                          \
      dense_of<uint8_t>(a[2], c10::ScalarType::Byte, num(a[4]) * groups(num(a[5]), num(a[6]))),                           \
      bytes(a[3], p_xnor_w4_wimg_bytes(num(a[4]), num(a[5]), num(a[6]))), num(a[4]), num(a[5]), num(a[6]))                \
    X(xnor_w4_linear, 9, rows(a[0], dtype(a[0]), num(a[4]), num(a[5])), stride(a[0], num(a[4]), num(a[5])),               \
      bytes(a[1], p_xnor_w4_wimg_bytes(num(a[6]), num(a[5]), num(a[7]))),                                                 \
      dense(a[2], scalar_type(dtype(a[0])), area(a[4], a[6])),                                                            \
      bytes(a[3], p_xnor_w4_linear_workspace_bytes(num(a[4]), num(a[5]), num(a[6]), num(a[7]))), num(a[4]), num(a[5]),    \
      num(a[6]), num(a[7]), dtype(a[0]))                                                                                  \
    X(xnor_w4_linear_q8, 11, dense_of<int8_t>(a[0], c10::ScalarType::Char, area(a[5], a[6])),                             \
      dense_f32(a[1], num(a[5]) * groups(num(a[6]), num(a[9]))),                                                          \
      bytes(a[2], p_xnor_w4_wimg_bytes(num(a[7]), num(a[6]), num(a[8]))),                                                 \
      dense(a[3], scalar_type(dtype(a[3])), area(a[5], a[7])),                                                            \
      bytes(a[4], p_xnor_w4_linear_workspace_bytes(num(a[5]), num(a[6]), num(a[7]), num(a[8]))), num(a[5]), num(a[6]),    \
      num(a[7]), num(a[8]), num(a[9]), dtype(a[3]))                                                                       \
    X(xnor_logprobs, 14, rows(a[0], dtype(a[0]), num(a[9]), num(a[10])), stride(a[0], num(a[9]), num(a[10])),             \
      tokens(a[1], area(a[9], a[11])), token_bytes(a[1]), dense_f32(a[2], area(a[9], a[11])), dense_f32(a[3], num(a[9])), \
      dense_f32(a[4], 2 * (int64_t)num(a[9])), dense_f32(a[5], num(a[9])),                                                \
      dense_of<int32_t>(a[6], c10::ScalarType::Int, area(a[9], a[12])), dense_f32(a[7], area(a[9], a[12])),               \
      bytes(a[8], p_xnor_logprobs_workspace_bytes(num(a[9]), num(a[10]), num(a[12]))), num(a[9]), num(a[10]), num(a[11]), \
      num(a[12]), dtype(a[0]))                                                                                            \
    X(xnor_logprobs_backward, 11, rows(a[0], dtype(a[0]), num(a[7]), num(a[8])), stride(a[0], num(a[7]), num(a[8])),      \
      tokens(a[1], area(a[7], a[9])), token_bytes(a[1]), dense_f32(a[2], 2 * (int64_t)num(a[7])),                         \
      dense_f32(a[3], num(a[7])), dense_f32(a[4], area(a[7], a[9])), dense_f32(a[5], num(a[7])),                          \
      dense(a[6], scalar_type(dtype(a[0])), area(a[7], a[8])), num(a[7]), num(a[8]), num(a[9]), dtype(a[0]))              \
    X(xnor_q8_rows, 7, rows(a[0], dtype(a[0]), num(a[3]), num(a[4])), stride(a[0], num(a[3]), num(a[4])),                 \
      dense_of<int8_t>(a[1], c10::ScalarType::Char, area(a[3], a[4])),                                                    \
      dense_f32(a[2], num(a[3]) * groups(num(a[4]), num(a[5]))), num(a[3]), num(a[4]), num(a[5]),                         \
      on_one_device(a, 7, dtype(a[0])))                                                                                   \
    X(xnor_w8_linear, 11, dense_of<int8_t>(a[0], c10::ScalarType::Char, area(a[7], a[8])), dense_f32(a[1], num(a[7])),    \
      dense_of<int8_t>(a[2], c10::ScalarType::Char, area(a[9], a[8])), dense_f32(a[3], num(a[9])),                        \
      dense_f32(a[4], num(a[9])), dense(a[5], scalar_type(dtype(a[5])), area(a[7], a[9])),                                \
      bytes(a[6], p_xnor_w8_linear_workspace_bytes(num(a[7]), num(a[8]), num(a[9]))), num(a[7]), num(a[8]), num(a[9]),    \
      on_one_device(a, 11, dtype(a[5])))                                                                                  \
    X(xnor_activation_q8, 13, rows(a[0], dtype(a[0]), num(a[6]), wide(a[7], a[11])),                                      \
      stride(a[0], num(a[6]), wide(a[7], a[11])), dense(a[1], scalar_type(dtype(a[0])), area(a[6], a[7])),                \
      dense_of<int8_t>(a[2], c10::ScalarType::Char, area(a[6], a[7])),                                                    \
      dense_f32(a[3], num(a[6]) * groups(num(a[7]), num(a[8]))),                                                          \
      dense_of<int8_t>(a[4], c10::ScalarType::Char, num(a[6]) * wide(a[7], a[11])),                                       \
      dense_f32(a[5], num(a[6]) * groups(wide(a[7], a[11]), num(a[9]))), num(a[6]), num(a[7]), num(a[8]), num(a[9]),      \
      num(a[10]), num(a[11]), on_one_device(a, 13, dtype(a[0])))                                                          \
    X(xnor_activation_backward, 10, dense_of<int8_t>(a[0], c10::ScalarType::Char, num(a[4]) * wide(a[5], a[8])),          \
      dense_f32(a[1], num(a[4]) * groups(wide(a[5], a[8]), num(a[6]))), rows(a[2], dtype(a[2]), num(a[4]), num(a[5])),    \
      stride(a[2], num(a[4]), num(a[5])), dense(a[3], scalar_type(dtype(a[2])), num(a[4]) * wide(a[5], a[8])), num(a[4]), \
      num(a[5]), num(a[6]), num(a[7]), num(a[8]), on_one_device(a, 10, dtype(a[2])))                                      \
    X(xnor_q8_weight_gradient, 12, dense_of<int8_t>(a[0], c10::ScalarType::Char, area(a[7], a[8])),                       \
      dense_f32(a[1], num(a[7]) * groups(num(a[8]), num(a[10]))), rows(a[2], dtype(a[2]), num(a[7]), num(a[9])),          \
      stride(a[2], num(a[7]), num(a[9])), dense(a[3], scalar_type(dtype(a[3])), area(a[9], a[8])),                        \
      dense_f32(a[4], num(a[9])), num(a[5]),                                                                              \
      bytes(a[6], p_xnor_q8_weight_gradient_workspace_bytes(num(a[7]), num(a[8]), num(a[9]), num(a[10]), dtype(a[2]),     \
                                                            dtype(a[3]))),                                                \
      num(a[7]), num(a[8]), num(a[9]), num(a[10]), dtype(a[2]), on_one_device(a, 12, dtype(a[3])))                        \
    X(xnor_sample, 13, rows(a[0], dtype(a[0]), num(a[10]), num(a[11])), stride(a[0], num(a[10]), num(a[11])),             \
      dense_f32(a[1], num(a[10])), dense_of<int32_t>(a[2], c10::ScalarType::Int, num(a[10])), dense_f32(a[3], num(a[10])),\
      dense_f32(a[4], num(a[10])), dense_f32(a[5], num(a[10])), dense_of<int32_t>(a[6], c10::ScalarType::Int, num(a[10])),\
      dense_f32(a[7], num(a[10])), dense_of<int32_t>(a[8], c10::ScalarType::Int, num(a[10])),                             \
      bytes(a[9], p_xnor_sample_workspace_bytes(num(a[10]), num(a[11]))), num(a[10]), num(a[11]),                         \
      on_one_device(a, 13, dtype(a[0])))

#define XNOR_POINTER(NAME, N, ...) decltype(&::NAME) p_##NAME = nullptr;
XNOR_CALLS(XNOR_POINTER)

// The C call itself runs without the interpreter's lock, as under ctypes: a launch can wait for room in its queue, and what
// empties the queue may be a host function that needs the lock.  A constructor, so that its braces convert the arguments in
// order; they come by reference, and descriptors live in the caller's full expression.
struct Enqueue {
    int status;
    template <class P, class... A> explicit Enqueue(P entry, A &&...args)
    {
        PyThreadState *state = PyEval_SaveThread();
        status = entry(args...);
        PyEval_RestoreThread(state);
    }
};

template <class F> PyObject *guarded(const char *name, F call)
{
    int status;
    try {
        status = call();
    } catch (const PythonError &) {
        return nullptr;
    } catch (const std::exception &e) {                  // (torch refuses the address of a tensor without storage)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    if (status == XNOR_OK) Py_RETURN_NONE;
    PyObject *r = PyObject_CallFunction(g_raise, "si", name, status);
    Py_XDECREF(r);
    if (r) PyErr_SetString(PyExc_RuntimeError, name);
    return nullptr;
}

#define XNOR_WRAPPER(NAME, N, ...)                                                                       \
    PyObject *call_##NAME(PyObject *, PyObject *const *a, Py_ssize_t n)                                  \
    {                                                                                                    \
        if (n != N || !p_##NAME) {                                                                       \
            PyErr_SetString(PyExc_TypeError, #NAME ": wrong number of arguments, or no library bound");  \
            return nullptr;                                                                              \
        }                                                                                                \
        return guarded(#NAME, [&] { return Enqueue{p_##NAME, __VA_ARGS__, stream(a[N - 1])}.status; });  \
    }
XNOR_CALLS(XNOR_WRAPPER)

// bind(path of the library, raise(name, status), current_device(), raw_stream(device), descriptor class)
PyObject *bind(PyObject *, PyObject *args)
{
    const char *path;
    PyObject *raise, *device, *raw, *desc;
    if (!PyArg_ParseTuple(args, "sOOOO", &path, &raise, &device, &raw, &desc)) return nullptr;
    void *lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!lib) {
        PyErr_SetString(PyExc_ImportError, dlerror());
        return nullptr;
    }
#define XNOR_LOOKUP(NAME, N, ...)                                                       \
    if (void *f = dlsym(lib, #NAME)) p_##NAME = reinterpret_cast<decltype(p_##NAME)>(f); \
    else {                                                                              \
        PyErr_SetString(PyExc_ImportError, #NAME " is not in the library");             \
        return nullptr;                                                                 \
    }
    XNOR_CALLS(XNOR_LOOKUP)
#define XNOR_QUERY_LOOKUP(NAME) XNOR_LOOKUP(NAME, 0)
    XNOR_QUERIES(XNOR_QUERY_LOOKUP)
    Py_INCREF(raise); Py_INCREF(device); Py_INCREF(raw); Py_INCREF(desc);
    Py_XDECREF(g_raise); Py_XDECREF(g_current_device); Py_XDECREF(g_raw_stream); Py_XDECREF(g_desc);
    g_raise = raise; g_current_device = device; g_raw_stream = raw; g_desc = desc;
    Py_RETURN_NONE;
}

#define XNOR_METHOD(NAME, N, ...) \
    {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call_##NAME)), METH_FASTCALL, nullptr},
PyMethodDef g_methods[] = {XNOR_CALLS(XNOR_METHOD){"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&g_module); }
