// The Python calls of the 8-bit matrices and of drawing candidates: argument
// checks, results' tensors and the current stream in C++.  A call that takes
// the GPU 3.5 us (a row through one layer) took the host 13.9 us in Python, most
// of it in attributes of tensors; it takes 5.6 so, half of it the launch.  Nothing
// is computed here, and nothing is kept from one call for the next but the
// addresses of the C functions.
//
// The functions take their arguments by position, in the order that hwsel.py
// passes them on.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <optional>
#include <utility>

#include "hwsel.h"

namespace {

struct Failed {};                                           // a Python error is set

struct Functions {
    decltype(&hwsel_fp8_quantise) quantise;
    decltype(&hwsel_fp8_dequantise) dequantise;
    decltype(&hwsel_fp8_transpose) transpose;
    decltype(&hwsel_fp8_matmul_workspace_bytes) matmul_workspace_bytes;
    decltype(&hwsel_fp8_matmul) matmul;
    decltype(&hwsel_fp8_layer) layer;
    decltype(&hwsel_sample_workspace_bytes) sample_workspace_bytes;
    decltype(&hwsel_sample_per_problem) sample;
    decltype(&hwsel_last_error) last_error;
} lib;
PyObject *error_class;                                      // HwselError
PyObject *k_q, *k_scale, *k_rows, *k_cols, *k_format, *k_block_rows, *k_stream;

// A reference owned here.
class Ref {
public:
    explicit Ref(PyObject *p = nullptr) : p_(p) {}
    Ref(Ref &&o) noexcept : p_(o.p_) { o.p_ = nullptr; }
    Ref &operator=(Ref &&o) noexcept
    {
        std::swap(p_, o.p_);
        return *this;
    }
    ~Ref() { Py_XDECREF(p_); }
    PyObject *get() const { return p_; }
    PyObject *release()
    {
        PyObject *p = p_;
        p_ = nullptr;
        return p;
    }

private:
    PyObject *p_;
};

PyObject *must(PyObject *p)
{
    if (!p) throw Failed{};
    return p;
}

template <class... T>
[[noreturn]] void refuse(const char *format, T... values)
{
    PyErr_Format(PyExc_ValueError, format, values...);
    throw Failed{};
}

void check(const char *fn, int status)
{
    if (status == HWSEL_OK) return;
    const Ref e(must(PyObject_CallFunction(error_class, "sis", fn, status, lib.last_error())));
    PyErr_SetObject(error_class, e.get());
    throw Failed{};
}

int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);                 // (what has an __index__, not a float)
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v;
}

int64_t entry(PyObject *m, PyObject *key) { return integer(Ref(must(PyObject_GetItem(m, key))).get()); }

int32_t int32_of(int64_t v, const char *name)
{
    if (v < INT32_MIN || v > INT32_MAX) refuse("%s: %lld is not a 32-bit number", name, (long long)v);
    return (int32_t)v;
}

hipStream_t stream_of(PyObject *stream)
{
    if (stream == Py_None) return c10::hip::getCurrentHIPStream().stream();
    const Ref number(PyLong_Check(stream) ? Py_NewRef(stream) : must(PyObject_GetAttr(stream, k_stream)));
    void *p = PyLong_AsVoidPtr(number.get());
    if (!p && PyErr_Occurred()) throw Failed{};
    return static_cast<hipStream_t>(p);
}

// The stream of a call, and what the call allocates.  torch hands memory that was
// freed to the next allocation of the same stream without waiting, so a call on
// another stream than the current one allocates on that one: nothing of the
// current stream still uses what it gets, and its workspace, freed on return,
// goes to later work of the same stream.  Results are the caller's, who uses
// them on the current stream: they are noted there too.
class Queue {
public:
    Queue(PyObject *given, int device) : device_(device), stream_(stream_of(given))
    {
        if (given == Py_None) return;
        const auto current = c10::hip::getCurrentHIPStream((c10::DeviceIndex)device);
        if (current.stream() == stream_) return;
        current_ = current;
        c10::hip::setCurrentHIPStream(c10::hip::getStreamFromExternal(stream_, (c10::DeviceIndex)device));
    }
    ~Queue()
    {
        if (current_) c10::hip::setCurrentHIPStream(*current_);
    }
    Queue(const Queue &) = delete;
    Queue &operator=(const Queue &) = delete;

    hipStream_t stream() const { return stream_; }
    at::Tensor workspace(int64_t bytes) const { return empty({bytes}, at::kByte); }
    at::Tensor result(at::IntArrayRef sizes, at::ScalarType type) const
    {
        at::Tensor t = empty(sizes, type);
        if (current_ && t.numel() != 0) c10::hip::HIPCachingAllocator::recordStream(t.storage().data_ptr(), *current_);
        return t;
    }

private:
    at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type) const
    {
        return at::empty(sizes, at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)device_));
    }

    int device_;
    hipStream_t stream_;
    std::optional<c10::hip::HIPStream> current_;            // torch's, where the call is on another
};

// A contiguous device tensor of dtype `type` with at least numel elements, on
// device `device` (-1: any).
const at::Tensor &argument(PyObject *o, const char *name, at::ScalarType type, int64_t numel, int device)
{
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda() || !THPVariable_Unpack(o).is_contiguous())
        refuse("%s must be a contiguous device tensor", name);
    const at::Tensor &t = THPVariable_Unpack(o);
    if (device >= 0 && t.get_device() != device)
        refuse("%s is on device %d, the other operands on %d", name, (int)t.get_device(), device);
    if (t.scalar_type() != type) refuse("%s has dtype %s, expected %s", name, c10::toString(t.scalar_type()), c10::toString(type));
    if (t.numel() < numel)
        refuse("%s holds %lld elements, the call needs %lld", name, (long long)t.numel(), (long long)numel);
    return t;
}

void *argument_or_null(PyObject *o, const char *name, at::ScalarType type, int64_t numel, int device)
{
    return o == Py_None ? nullptr : argument(o, name, type, numel, device).data_ptr();
}

// A row-major fp32 or bf16 matrix of at least rows x cols on `device`.
struct Plain {
    void *data;
    int32_t dtype;
    int64_t rows, cols, ld;
};

int32_t dtype_code(at::ScalarType t, const char *name)
{
    if (t != at::kBFloat16 && t != at::kFloat) refuse("%s must be fp32 or bf16, not %s", name, c10::toString(t));
    return t == at::kFloat ? HWSEL_DTYPE_FP32 : HWSEL_DTYPE_BF16;
}

// The step between rows goes on as it is where there are several: a matrix whose
// rows overlap (an unfold view, say) is refused, not read at another step.
Plain plain(const at::Tensor &t, const char *name, int64_t rows, int64_t cols, int device)
{
    if (!t.is_cuda() || t.dim() != 2 || t.get_device() != device) refuse("%s must be a 2-D device tensor on device %d", name, device);
    const int32_t code = dtype_code(t.scalar_type(), name);
    const int64_t r = t.size(0), c = t.size(1), step = t.stride(0);
    if ((c > 1 && t.stride(1) != 1) || r < rows || c < cols || (r > 1 && step < c))
        refuse("%s must be at least [%lld][%lld], with unit column stride and rows that do not overlap", name, (long long)rows, (long long)cols);
    return {t.data_ptr(), code, r, c, r > 1 ? step : c};    // (torch gives the step of a single row any value)
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) refuse("%s must be a 2-D device tensor", name);
    return THPVariable_Unpack(o);
}

// An 8-bit matrix: what the C functions take, and its device.
struct Fp8 {
    hwsel_fp8_t c;
    int device;
};

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

Fp8 fp8(PyObject *m, const char *name, int device = -1)
{
    const Ref q_ref(must(PyObject_GetItem(m, k_q))), s_ref(must(PyObject_GetItem(m, k_scale)));
    const int64_t rows = entry(m, k_rows), cols = entry(m, k_cols), block_rows = entry(m, k_block_rows), format = entry(m, k_format);
    if (rows < 1 || cols < 1) refuse("%s: %lld x %lld", name, (long long)rows, (long long)cols);
    const struct {
        PyObject *o;
        const char *part;
    } parts[2] = {{q_ref.get(), "q"}, {s_ref.get(), "scale"}};
    for (const auto &p : parts) {
        if (!THPVariable_Check(p.o)) refuse("%s.%s must be a 2-D uint8 device tensor with unit column stride", name, p.part);
        const at::Tensor &t = THPVariable_Unpack(p.o);
        if (!t.is_cuda() || t.dim() != 2 || t.scalar_type() != at::kByte || (t.stride(1) != 1 && t.size(1) > 1))
            refuse("%s.%s must be a 2-D uint8 device tensor with unit column stride", name, p.part);
        if (device < 0) device = t.get_device();
        if (t.get_device() != device)
            refuse("%s.%s is on device %d, the other operands on %d", name, p.part, (int)t.get_device(), device);
    }
    const at::Tensor &q = THPVariable_Unpack(q_ref.get()), &s = THPVariable_Unpack(s_ref.get());
    const int64_t width = up(cols, HWSEL_FP8_BLOCK), words = up(width / HWSEL_FP8_BLOCK, 4), high = block_rows > 1 ? block_rows : 1;
    if (q.size(0) < rows || q.size(1) < width || s.size(0) < (rows + high - 1) / high || s.size(1) < words)
        refuse("%s: buffers [%lld][%lld], [%lld][%lld] are short of %lld x %lld", name, (long long)q.size(0), (long long)q.size(1),
               (long long)s.size(0), (long long)s.size(1), (long long)rows, (long long)cols);
    // (the step of a single row is never taken, and torch gives it any value)
    return {{rows, cols, static_cast<uint8_t *>(q.data_ptr()), q.size(0) > 1 ? q.stride(0) : width,
             static_cast<uint8_t *>(s.data_ptr()), s.size(0) > 1 ? s.stride(0) : words, int32_of(format, "format"),
             int32_of(block_rows, "block_rows")},
            device};
}

// Buffers of an 8-bit matrix as a dict, and what the C functions take.
PyObject *fp8_empty(int64_t rows, int64_t cols, int64_t format, int64_t block_rows, const Queue &queue, int device, Fp8 &to)
{
    if (rows < 1 || cols < 1) refuse("a matrix of %lld x %lld", (long long)rows, (long long)cols);
    const int64_t width = up(cols, HWSEL_FP8_BLOCK), words = up(width / HWSEL_FP8_BLOCK, 4), high = block_rows > 1 ? block_rows : 1;
    const at::Tensor q = queue.result({rows, width}, at::kByte), s = queue.result({(rows + high - 1) / high, words}, at::kByte);
    to = {{rows, cols, static_cast<uint8_t *>(q.data_ptr()), width, static_cast<uint8_t *>(s.data_ptr()), words,
           int32_of(format, "format"), int32_of(block_rows, "block_rows")},
          device};
    Ref d(must(PyDict_New()));
    auto put = [&](PyObject *key, PyObject *value) {
        const Ref v(must(value));
        if (PyDict_SetItem(d.get(), key, v.get()) != 0) throw Failed{};
    };
    put(k_q, THPVariable_Wrap(q));
    put(k_scale, THPVariable_Wrap(s));
    put(k_rows, PyLong_FromLongLong(rows));
    put(k_cols, PyLong_FromLongLong(cols));
    put(k_format, PyLong_FromLongLong(format));
    put(k_block_rows, PyLong_FromLongLong(block_rows));
    return d.release();
}

PyObject *keep(PyObject *o)
{
    Py_INCREF(o);
    return o;
}

// Device memory for a call: the caller's, or some of this call's own.
struct Workspace {
    at::Tensor own;
    void *data = nullptr;
    size_t bytes = 0;
};

Workspace workspace_of(PyObject *given, size_t need, const Queue &queue, int device)
{
    Workspace w;
    if (given != Py_None) {
        const at::Tensor &t = argument(given, "workspace", at::kByte, 0, device);
        w.data = t.data_ptr();
        w.bytes = (size_t)t.numel();
    } else if (need != 0) {
        w.own = queue.workspace((int64_t)need);
        w.data = w.own.data_ptr();
        w.bytes = need;
    }
    return w;
}

Workspace product_workspace(PyObject *given, const Fp8 &a, const Fp8 &b, const Queue &queue)
{
    size_t need = 0;
    if (given == Py_None) check("hwsel_fp8_matmul_workspace_bytes", lib.matmul_workspace_bytes(&a.c, &b.c, &need));
    return workspace_of(given, need, queue, a.device);
}

// (X, format, block_rows, transpose, mean, inv_std, out, stream)
PyObject *quantise(PyObject *const *v)
{
    const at::Tensor &X = tensor(v[0], "X");
    const Plain x = plain(X, "X", 1, 1, X.is_cuda() ? X.get_device() : 0);
    const int device = X.get_device();
    const Queue queue(v[7], device);
    const int64_t format = integer(v[1]), block_rows = integer(v[2]);
    const int transpose = PyObject_IsTrue(v[3]);
    if (transpose < 0) throw Failed{};
    const int64_t rows = transpose ? x.cols : x.rows, cols = transpose ? x.rows : x.cols;
    const auto *mean = static_cast<const float *>(argument_or_null(v[4], "mean", at::kFloat, x.cols, device));
    const auto *inv_std = static_cast<const float *>(argument_or_null(v[5], "inv_std", at::kFloat, x.cols, device));
    Fp8 to;
    Ref out;
    if (v[6] == Py_None) {
        out = Ref(fp8_empty(rows, cols, format, block_rows, queue, device, to));
    } else {
        to = fp8(v[6], "out", device);
        if (to.c.rows != rows || to.c.cols != cols || to.c.format != format || to.c.block_rows != block_rows)
            refuse("out is not a %lld x %lld matrix of this format and block_rows", (long long)rows, (long long)cols);
        out = Ref(keep(v[6]));
    }
    check("hwsel_fp8_quantise", lib.quantise(x.data, x.dtype, x.ld, transpose, mean, inv_std, &to.c, queue.stream()));
    return out.release();
}

at::ScalarType dtype_of(PyObject *o)
{
    if (!THPDtype_Check(o)) refuse("dtype must be torch.float32 or torch.bfloat16");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

// The caller's matrix for a result, or a new one.
Plain result(PyObject *given, int64_t rows, int64_t cols, PyObject *dtype, const Queue &queue, int device, Ref &out)
{
    if (given != Py_None) {
        out = Ref(keep(given));
        return plain(tensor(given, "out"), "out", rows, cols, device);
    }
    const at::ScalarType type = dtype_of(dtype);
    const int32_t code = dtype_code(type, "out");
    const at::Tensor t = queue.result({rows, cols}, type);
    out = Ref(must(THPVariable_Wrap(t)));
    return {t.data_ptr(), code, rows, cols, cols};
}

// (m, dtype, out, stream)
PyObject *dequantise(PyObject *const *v)
{
    const Fp8 m = fp8(v[0], "m");
    const Queue queue(v[3], m.device);
    Ref out;
    const Plain to = result(v[2], m.c.rows, m.c.cols, v[1], queue, m.device, out);
    check("hwsel_fp8_dequantise", lib.dequantise(&m.c, to.data, to.dtype, to.ld, queue.stream()));
    return out.release();
}

// (m, format, block_rows, out, stream)
PyObject *transpose(PyObject *const *v)
{
    const Fp8 m = fp8(v[0], "m");
    const Queue queue(v[4], m.device);
    Fp8 to;
    Ref out;
    if (v[3] == Py_None) {
        out = Ref(fp8_empty(m.c.cols, m.c.rows, integer(v[1]), integer(v[2]), queue, m.device, to));
    } else {
        to = fp8(v[3], "out", m.device);
        out = Ref(keep(v[3]));
    }
    check("hwsel_fp8_transpose", lib.transpose(&m.c, &to.c, queue.stream()));
    return out.release();
}

int activation(PyObject *gelu)
{
    const int on = PyObject_IsTrue(gelu);
    if (on < 0) throw Failed{};
    return on ? HWSEL_ACT_GELU : HWSEL_ACT_NONE;
}

// (A, B)
PyObject *matmul_workspace_bytes(PyObject *const *v)
{
    const Fp8 a = fp8(v[0], "A"), b = fp8(v[1], "B");
    size_t need = 0;
    check("hwsel_fp8_matmul_workspace_bytes", lib.matmul_workspace_bytes(&a.c, &b.c, &need));
    return must(PyLong_FromSize_t(need));
}

// (A, B, dtype, bias, gelu, out, workspace, stream)
PyObject *matmul(PyObject *const *v)
{
    const Fp8 a = fp8(v[0], "A"), b = fp8(v[1], "B", a.device);
    const Queue queue(v[7], a.device);
    Ref out;
    const Plain to = result(v[5], a.c.rows, b.c.rows, v[2], queue, a.device, out);
    const auto *bias = static_cast<const float *>(argument_or_null(v[3], "bias", at::kFloat, b.c.rows, a.device));
    const Workspace w = product_workspace(v[6], a, b, queue);
    check("hwsel_fp8_matmul", lib.matmul(&a.c, &b.c, bias, activation(v[4]), to.data, to.dtype, to.ld, w.data, w.bytes, queue.stream()));
    return out.release();
}

// (A, B, bias, gelu, out, workspace, stream)
PyObject *layer(PyObject *const *v)
{
    const Fp8 a = fp8(v[0], "A"), b = fp8(v[1], "B", a.device);
    const Queue queue(v[6], a.device);
    Fp8 to;
    Ref out;
    if (v[4] == Py_None) {
        out = Ref(fp8_empty(a.c.rows, b.c.rows, HWSEL_FP8_E4M3, 1, queue, a.device, to));
    } else {
        to = fp8(v[4], "out", a.device);
        out = Ref(keep(v[4]));
    }
    const auto *bias = static_cast<const float *>(argument_or_null(v[2], "bias", at::kFloat, b.c.rows, a.device));
    const Workspace w = product_workspace(v[5], a, b, queue);
    check("hwsel_fp8_layer", lib.layer(&a.c, &b.c, bias, activation(v[3]), &to.c, w.data, w.bytes, queue.stream()));
    return out.release();
}

// A setting of every problem, or one number: to the pointer or the number.
void setting(PyObject *o, const char *name, int64_t P, int device, float &number, const float *&each)
{
    if (THPVariable_Check(o)) {
        each = static_cast<const float *>(argument(o, name, at::kFloat, P, device).data_ptr());
        return;
    }
    const double d = PyFloat_AsDouble(o);
    if (d == -1.0 && PyErr_Occurred()) throw Failed{};
    number = (float)d;
}

// (scores, seg_offsets, u, temperature, top_k, top_p, min_p, idx, prob, kept, workspace, stream)
PyObject *sample(PyObject *const *v)
{
    const at::Tensor &scores = argument(v[0], "scores", at::kFloat, 0, -1);
    const int device = scores.get_device();
    const Queue queue(v[11], device);
    const at::Tensor &seg = argument(v[1], "seg_offsets", at::kLong, 2, device);
    const at::Tensor &u = argument(v[2], "u", at::kFloat, 0, device);
    const int64_t P = seg.size(0) - 1, R = scores.numel();
    if (u.dim() != 2 || u.size(0) != P) refuse("u must be [%lld][draws]", (long long)P);
    const int64_t draws = u.size(1);
    const int32_t p32 = int32_of(P, "problems"), draws32 = int32_of(draws, "draws");
    hwsel_sampling_t how{};
    setting(v[3], "temperature", P, device, how.temperature, how.temperature_of);
    if (THPVariable_Check(v[4])) {
        how.top_k_of = static_cast<const int32_t *>(argument(v[4], "top_k", at::kInt, P, device).data_ptr());
    } else {
        const int64_t k = integer(v[4]);                    // (past 2^31 - 1: all, as that is)
        how.top_k = (int32_t)(k > INT32_MAX ? INT32_MAX : k < 0 ? 0 : k);
    }
    setting(v[5], "top_p", P, device, how.top_p, how.top_p_of);
    setting(v[6], "min_p", P, device, how.min_p, how.min_p_of);
    auto out = [&](PyObject *given, const char *name, at::ScalarType type, at::IntArrayRef sizes, int64_t numel, void *&data) {
        if (given != Py_None) {
            data = argument(given, name, type, numel, device).data_ptr();
            return Ref(keep(given));
        }
        const at::Tensor t = queue.result(sizes, type);
        data = t.data_ptr();
        return Ref(must(THPVariable_Wrap(t)));
    };
    void *idx_at, *prob_at, *kept_at;
    const Ref idx = out(v[7], "idx", at::kInt, {P, draws}, P * draws, idx_at), prob = out(v[8], "prob", at::kFloat, {P, draws}, P * draws, prob_at),
              kept = out(v[9], "kept", at::kInt, {P}, P, kept_at);
    size_t need = 0;
    check("hwsel_sample_workspace_bytes", lib.sample_workspace_bytes(R, p32, draws32, &need));
    if (v[10] != Py_None) argument(v[10], "workspace", at::kByte, (int64_t)need, device);
    const Workspace w = workspace_of(v[10], need, queue, device);
    check("hwsel_sample_per_problem",
          lib.sample(static_cast<const float *>(scores.data_ptr()), R, static_cast<const int64_t *>(seg.data_ptr()), p32, &how,
                     static_cast<const float *>(u.data_ptr()), draws32, static_cast<int32_t *>(idx_at), static_cast<float *>(prob_at),
                     static_cast<int32_t *>(kept_at), w.data, w.bytes, queue.stream()));
    return must(PyTuple_Pack(3, idx.get(), prob.get(), kept.get()));
}

template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (!error_class || n != N) {
        PyErr_Format(PyExc_RuntimeError, error_class ? "%zd arguments expected, %zd given" : "not connected to the library", N, n);
        return nullptr;
    }
    HANDLE_TH_ERRORS
    try {
        return F(args);
    } catch (const Failed &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// connect(HwselError, address of each function in the order of Functions).
PyObject *connect(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    constexpr Py_ssize_t kFunctions = sizeof(Functions) / sizeof(void *);
    if (n != 1 + kFunctions) {
        PyErr_Format(PyExc_RuntimeError, "%zd arguments expected, %zd given", 1 + kFunctions, n);
        return nullptr;
    }
    void *at[kFunctions];
    for (Py_ssize_t i = 0; i < kFunctions; ++i) {
        at[i] = PyLong_AsVoidPtr(args[1 + i]);
        if (!at[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "a function is missing");
            return nullptr;
        }
    }
    static_assert(sizeof at == sizeof lib, "addresses alone");
    memcpy(&lib, at, sizeof lib);
    error_class = keep(args[0]);
    Py_RETURN_NONE;
}

template <class F>
constexpr PyCFunction entry_of(F *f)
{
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {
    {"connect", entry_of(connect), METH_FASTCALL, nullptr},
    {"fp8_quantise", entry_of(call<quantise, 8>), METH_FASTCALL, nullptr},
    {"fp8_dequantise", entry_of(call<dequantise, 4>), METH_FASTCALL, nullptr},
    {"fp8_transpose", entry_of(call<transpose, 5>), METH_FASTCALL, nullptr},
    {"fp8_matmul_workspace_bytes", entry_of(call<matmul_workspace_bytes, 2>), METH_FASTCALL, nullptr},
    {"fp8_matmul", entry_of(call<matmul, 8>), METH_FASTCALL, nullptr},
    {"fp8_layer", entry_of(call<layer, 7>), METH_FASTCALL, nullptr},
    {"sample_per_problem", entry_of(call<sample, 12>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Calls of libhwsel.so that are made in C++.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding()
{
    const struct {
        PyObject **key;
        const char *text;
    } keys[] = {{&k_q, "q"}, {&k_scale, "scale"}, {&k_rows, "rows"}, {&k_cols, "cols"}, {&k_format, "format"},
                {&k_block_rows, "block_rows"}, {&k_stream, "cuda_stream"}};
    for (const auto &k : keys)
        if (!(*k.key = PyUnicode_InternFromString(k.text))) return nullptr;
    return PyModule_Create(&module);
}
