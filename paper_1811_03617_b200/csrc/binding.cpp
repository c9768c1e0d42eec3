// The short way from Python to the entry points that a step calls once per product: their checks, allocations and calls in one function
// each, which takes tensors as they are.  Whatever is not plainly right (another type, size or device, an error of the call) is not
// dealt with here: the function says so by returning None or False, and gvq.py goes its own way, which names what is wrong.  With small
// operands the host's part is the whole of a call's time: i8_quantize 7.5 us through ctypes, i8_matmul 5.2, of which 2.2 and 2.8 are the
// launch's.
// Arguments are unpacked with the interpreter's lock, and the call and its allocations run without it: a launch waits where the stream's
// queue is full, which may be emptied by another Python thread alone (a host function in the stream), and an allocation may wait for
// the device.  Calls of one context take turns: its stream is set for each.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <mutex>
#include <utility>

#include "gvq.h"

namespace {

struct {
    decltype(&gvq_set_stream) set_stream;
    decltype(&gvq_i8_scratch_bytes) i8_scratch_bytes;
    decltype(&gvq_i8_quantize) i8_quantize;
    decltype(&gvq_i8_matmul) i8_matmul;
    decltype(&gvq_i8_gated) i8_gated;
    decltype(&gvq_gated_workspace_bytes) gated_workspace_bytes;
    decltype(&gvq_gated_forward) gated_forward;
    decltype(&gvq_gated_backward) gated_backward;
} entry = {};

// The class of quantized matrices and where its slots lie in an object.
PyTypeObject *i8_type = nullptr;
enum { kRows, kCols, kDevice, kCodes, kScales, kBuf, kCodesPtr, kScalesPtr, kSlots };
const char *const slot_names[kSlots] = {"rows", "cols", "device", "_codes", "_scales", "_buf", "codes_ptr", "scales_ptr"};
Py_ssize_t slot_at[kSlots];

PyObject *&slot(PyObject *o, int i) { return *reinterpret_cast<PyObject **>(reinterpret_cast<char *>(o) + slot_at[i]); }

// Without the interpreter's lock from here to the end of the block.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked &) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

struct Context {
    gvq_ctx *h;
    int device;
    // The context's stream becomes torch's current one.
    bool ready() const { return entry.set_stream(h, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()) == GVQ_OK; }
    // What its calls take in turn, without the interpreter's lock; contexts may share one.
    std::mutex &turn() const
    {
        static std::mutex turns[16];
        return turns[(reinterpret_cast<uintptr_t>(h) >> 6) % 16];
    }
};
// A context's handle and device.
bool open(PyObject *handle, PyObject *device, Context &c)
{
    c.h = static_cast<gvq_ctx *>(PyLong_AsVoidPtr(handle));
    c.device = (int)PyLong_AsLong(device);
    return c.h && entry.set_stream && !PyErr_Occurred();
}

struct Matrix {
    void *p;
    int64_t rows, cols, ld;
    int dtype;
};
int code_of(at::ScalarType t)
{
    return t == at::kFloat ? GVQ_F32 : t == at::kBFloat16 ? GVQ_BF16 : t == at::kHalf ? GVQ_F16 : -1;
}
bool matrix(PyObject *o, int device, Matrix &m)
{
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || t.dim() != 2 || !t.is_cuda() || t.get_device() != device || t.is_neg() || t.is_conj()) return false;
    m.rows = t.size(0);
    m.cols = t.size(1);
    if (m.rows < 1 || m.cols < 1 || (m.cols > 1 && t.stride(1) != 1)) return false;
    m.ld = m.rows > 1 ? t.stride(0) : m.cols;
    m.dtype = code_of(t.scalar_type());
    m.p = t.data_ptr();
    return m.dtype >= 0;
}
bool matrix(PyObject *o, int device, Matrix &m, int64_t rows, int64_t cols, int dtype)
{
    return matrix(o, device, m) && m.rows == rows && m.cols == cols && m.dtype == dtype;
}
bool aligned(const Matrix &m) { return (reinterpret_cast<uintptr_t>(m.p) & 15) == 0 && (m.rows == 1 || m.ld % 8 == 0); }

at::Tensor room(int64_t bytes, int device)
{
    return at::detail::empty_cuda({bytes}, at::kByte, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), c10::nullopt);
}

struct Quantized {
    int64_t rows, cols;
    int8_t *codes;
    float *scales;
};
bool quantized(PyObject *o, int device, Quantized &q)
{
    if (Py_TYPE(o) != i8_type) return false;
    for (int i : {kRows, kCols, kDevice, kCodesPtr, kScalesPtr})
        if (!slot(o, i)) return false;
    q.rows = PyLong_AsLongLong(slot(o, kRows));
    q.cols = PyLong_AsLongLong(slot(o, kCols));
    q.codes = static_cast<int8_t *>(PyLong_AsVoidPtr(slot(o, kCodesPtr)));
    q.scales = static_cast<float *>(PyLong_AsVoidPtr(slot(o, kScalesPtr)));
    return PyLong_AsLong(slot(o, kDevice)) == device;
}
// A reference that is given up unless it is taken.
struct Ref {
    PyObject *o = nullptr;
    Ref() = default;
    explicit Ref(PyObject *p) : o(p) {}
    Ref(const Ref &) = delete;
    Ref &operator=(Ref &&r)
    {
        std::swap(o, r.o);
        return *this;
    }
    ~Ref() { Py_XDECREF(o); }
    PyObject *take() { return std::exchange(o, nullptr); }
};
// An object whose slots are these; what it held before is given up.
void fill(PyObject *o, int64_t rows, int64_t cols, int device, PyObject *codes, PyObject *scales, PyObject *buf, const void *codes_at,
          const void *scales_at)
{
    PyObject *v[kSlots] = {PyLong_FromLongLong(rows), PyLong_FromLongLong(cols), PyLong_FromLong(device), Py_NewRef(codes), Py_NewRef(scales), buf,
                           PyLong_FromVoidPtr(const_cast<void *>(codes_at)), PyLong_FromVoidPtr(const_cast<void *>(scales_at))};
    for (int i = 0; i < kSlots; ++i) {
        PyObject *old = std::exchange(slot(o, i), v[i]);
        Py_XDECREF(old);
    }
}

// Room for a matrix, codes and scales in one allocation; the object of such a matrix.
at::Tensor room_for(int64_t rows, int64_t cols, int device, Quantized &q)
{
    const int64_t at = (rows * ((cols + 15) / 16 * 16) + 255) / 256 * 256;
    at::Tensor buf = room(at + 4 * rows, device);
    q = {rows, cols, static_cast<int8_t *>(buf.data_ptr()), reinterpret_cast<float *>(static_cast<char *>(buf.data_ptr()) + at)};
    return buf;
}
PyObject *new_quantized(const Quantized &q, int device, at::Tensor &&buf)
{
    PyObject *o = i8_type->tp_alloc(i8_type, 0);
    if (o) fill(o, q.rows, q.cols, device, Py_None, Py_None, THPVariable_Wrap(std::move(buf)), q.codes, q.scales);
    return o;
}

// Errors of what is called on the way (a Python error of a conversion, no memory) are the long way's to raise.
template <typename F>
PyObject *guarded(F f)
{
    PyObject *r = nullptr;
    try {
        r = f();
    } catch (...) {
    }
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_CLEAR(r);
    }
    return r ? r : Py_NewRef(Py_None);
}
PyObject *truth(bool b) { return Py_NewRef(b ? Py_True : Py_False); }
// What f, a call of the context that touches no Python object, says.
template <typename F>
PyObject *without_lock(const Context &c, F f)
{
    bool done;
    {
        Unlocked unlocked;
        const std::lock_guard<std::mutex> hold(c.turn());
        done = c.ready() && f();
    }
    return truth(done);
}

// bind(addresses of the entry points in the order above, the class of quantized matrices)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    constexpr int kEntries = sizeof(entry) / sizeof(void *);
    if (n != kEntries + 1 || !PyType_Check(args[kEntries])) {
        PyErr_SetString(PyExc_TypeError, "bind: the entry points and the class are wanted");
        return nullptr;
    }
    PyTypeObject *type = reinterpret_cast<PyTypeObject *>(args[kEntries]);
    for (int i = 0; i < kSlots; ++i) {
        PyObject *d = PyDict_GetItemString(type->tp_dict, slot_names[i]);
        if (!d || !Py_IS_TYPE(d, &PyMemberDescr_Type)) {
            PyErr_Format(PyExc_TypeError, "bind: the class has no slot %s", slot_names[i]);
            return nullptr;
        }
        slot_at[i] = reinterpret_cast<PyMemberDescrObject *>(d)->d_member->offset;
    }
    void *p[kEntries];
    for (int i = 0; i < kEntries; ++i)
        if (!(p[i] = PyLong_AsVoidPtr(args[i]))) return nullptr;
    memcpy(&entry, p, sizeof(entry));
    Py_XINCREF(type);
    i8_type = type;
    return Py_NewRef(Py_None);
}

// i8_fill(matrix, rows, columns, codes, scales): whether the matrix is now of these codes and scales
PyObject *i8_fill(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 5 || Py_TYPE(args[0]) != i8_type || !PyLong_CheckExact(args[1]) || !PyLong_CheckExact(args[2]) || !THPVariable_Check(args[3]) ||
            !THPVariable_Check(args[4]))
            return nullptr;
        const int64_t rows = PyLong_AsLongLong(args[1]), cols = PyLong_AsLongLong(args[2]);
        if (rows < 1 || cols < 1 || rows > INT32_MAX - 1024 || cols > INT32_MAX - 1024 || (rows + 127) / 128 >= INT32_MAX / ((cols + 127) / 128))
            return nullptr;
        const at::Tensor &codes = THPVariable_Unpack(args[3]), &scales = THPVariable_Unpack(args[4]);
        for (const at::Tensor *t : {&codes, &scales})
            if (t->layout() != at::kStrided || !t->is_cuda() || !t->is_contiguous() || t->is_neg()) return nullptr;
        if (codes.scalar_type() != at::kChar || scales.scalar_type() != at::kFloat || codes.numel() != rows * ((cols + 15) / 16 * 16) ||
            scales.numel() != rows || codes.get_device() != scales.get_device())
            return nullptr;
        fill(args[0], rows, cols, codes.get_device(), args[3], args[4], nullptr, codes.data_ptr(), scales.data_ptr());
        return truth(true);
    });
}

// i8_quantize(handle, device, x, by rows, by columns, stochastic, seed, node): the matrix or matrices, or None
PyObject *i8_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Context c;
        Matrix x;
        if (n != 8 || !open(args[0], args[1], c) || !matrix(args[2], c.device, x)) return nullptr;
        const bool by_rows = args[3] == Py_True, by_cols = args[4] == Py_True;
        const int stochastic = PyObject_IsTrue(args[5]);
        const uint64_t seed = PyLong_AsUnsignedLongLongMask(args[6]);
        const uint32_t node = (uint32_t)PyLong_AsUnsignedLongMask(args[7]);
        if (PyErr_Occurred() || x.rows > INT32_MAX - 1024 || x.cols > INT32_MAX - 1024) return nullptr;
        Quantized q = {}, t = {};
        at::Tensor buf, buf_t;
        {
            Unlocked unlocked;
            const std::lock_guard<std::mutex> hold(c.turn());
            if (!c.ready()) return nullptr;
            if (by_rows) buf = room_for(x.rows, x.cols, c.device, q);
            if (by_cols) buf_t = room_for(x.cols, x.rows, c.device, t);
            const int64_t bytes = by_cols ? entry.i8_scratch_bytes(x.rows, x.cols) : 0;
            at::Tensor scratch;
            if (bytes > 0) scratch = room(bytes, c.device);
            if (bytes < 0 || entry.i8_quantize(c.h, x.p, x.dtype, x.rows, x.cols, x.ld, stochastic, seed, node, q.codes, q.scales, t.codes, t.scales,
                                               bytes > 0 ? scratch.data_ptr() : nullptr, (size_t)bytes) != GVQ_OK)
                return nullptr;
        }
        Ref out, out_t;
        if (by_rows) out = Ref(new_quantized(q, c.device, std::move(buf)));
        if (by_cols) out_t = Ref(new_quantized(t, c.device, std::move(buf_t)));
        if ((by_rows && !out.o) || (by_cols && !out_t.o)) return nullptr;
        return by_rows && by_cols ? PyTuple_Pack(2, out.o, out_t.o) : by_rows ? out.take() : out_t.take();
    });
}

// i8_matmul(handle, device, a, b, out): whether it was done
PyObject *i8_matmul(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Context c;
        Quantized a, b;
        Matrix out;
        if (n != 5 || !open(args[0], args[1], c) || !quantized(args[2], c.device, a) || !quantized(args[3], c.device, b) ||
            !matrix(args[4], c.device, out) || a.cols != b.cols || out.rows != a.rows || out.cols != b.rows)
            return nullptr;
        return without_lock(c, [&] {
            return entry.i8_matmul(c.h, a.codes, a.scales, b.codes, b.scales, a.rows, b.rows, a.cols, out.p, out.dtype, out.ld) == GVQ_OK;
        });
    });
}

// i8_gated(handle, device, a, gate, up, out, activation): whether it was done
PyObject *i8_gated(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Context c;
        Quantized a, g, u;
        Matrix out;
        if (n != 7 || !open(args[0], args[1], c) || !quantized(args[2], c.device, a) || !quantized(args[3], c.device, g) ||
            !quantized(args[4], c.device, u) || !matrix(args[5], c.device, out) || a.cols != g.cols || a.cols != u.cols || g.rows != u.rows ||
            out.rows != a.rows || out.cols != g.rows)
            return nullptr;
        const int act = (int)PyLong_AsLong(args[6]);
        if (PyErr_Occurred()) return nullptr;
        return without_lock(c, [&] {
            return entry.i8_gated(c.h, a.codes, a.scales, g.codes, g.scales, u.codes, u.scales, a.rows, g.rows, a.cols, act, out.p,
                                               out.dtype, out.ld) == GVQ_OK;
        });
    });
}

// gated_forward(handle, device, x, w_gate, w_up, out, activation, gate or None, up or None): whether it was done
PyObject *gated_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Context c;
        Matrix x, wg, wu, h, g = {}, u = {};
        if (n != 9 || !open(args[0], args[1], c) || !matrix(args[2], c.device, x) || x.dtype == GVQ_F32 || !matrix(args[3], c.device, wg) ||
            wg.cols != x.cols || wg.dtype != x.dtype || !matrix(args[4], c.device, wu, wg.rows, wg.cols, x.dtype) ||
            !matrix(args[5], c.device, h, x.rows, wg.rows, x.dtype) || (args[7] == Py_None) != (args[8] == Py_None))
            return nullptr;
        if (args[7] != Py_None && (!matrix(args[7], c.device, g, h.rows, h.cols, x.dtype) || !matrix(args[8], c.device, u, h.rows, h.cols, x.dtype)))
            return nullptr;
        const int act = (int)PyLong_AsLong(args[6]);
        if (PyErr_Occurred()) return nullptr;
        return without_lock(c, [&] {
            const int64_t bytes = aligned(x) && aligned(wg) && aligned(wu) ? 0 : entry.gated_workspace_bytes(x.rows, wg.rows, x.cols, 0, 0);
            if (bytes < 0) return false;
            at::Tensor ws;
            if (bytes > 0) ws = room(bytes, c.device);
            return entry.gated_forward(c.h, x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld, x.dtype, x.rows, wg.rows, x.cols, act, h.p, h.ld, g.p, g.ld, u.p, u.ld,
                                       bytes > 0 ? ws.data_ptr() : nullptr, (size_t)bytes) == GVQ_OK;
        });
    });
}

// gated_backward(handle, device, dh, gate, up, x, w_gate, w_up, activation, dx, dw_gate, dw_up; None where not given): whether it was done
PyObject *gated_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        Context c;
        Matrix dh, g, u, x = {}, wg = {}, wu = {}, dx = {}, dg = {}, du = {};
        if (n != 12 || !open(args[0], args[1], c) || !matrix(args[2], c.device, dh) || dh.dtype == GVQ_F32 ||
            !matrix(args[3], c.device, g, dh.rows, dh.cols, dh.dtype) || !matrix(args[4], c.device, u, dh.rows, dh.cols, dh.dtype))
            return nullptr;
        const int64_t M = dh.rows, F = dh.cols;
        const bool want_x = args[9] != Py_None, want_g = args[10] != Py_None, want_u = args[11] != Py_None;
        int64_t K = 0;
        bool plain = true;
        if (want_x) {
            if (!matrix(args[9], c.device, dx)) return nullptr;
            K = dx.cols;
            if (dx.rows != M || dx.dtype != dh.dtype || !matrix(args[6], c.device, wg, F, K, dh.dtype) || !matrix(args[7], c.device, wu, F, K, dh.dtype))
                return nullptr;
            plain = aligned(wg) && aligned(wu);
        }
        if (want_g || want_u) {
            if ((want_g && !matrix(args[10], c.device, dg)) || (want_u && !matrix(args[11], c.device, du))) return nullptr;
            const Matrix &d = want_g ? dg : du;
            if (!want_x) K = d.cols;
            if (d.rows != F || d.cols != K || (want_g && want_u && (du.rows != F || du.cols != K || du.dtype != dg.dtype)) ||
                !matrix(args[5], c.device, x, M, K, dh.dtype))
                return nullptr;
            plain = plain && aligned(x);
        }
        if (!K) return nullptr;
        const int act = (int)PyLong_AsLong(args[8]);
        if (act < 0 || PyErr_Occurred()) return nullptr;
        return without_lock(c, [&] {
            const int64_t bytes = entry.gated_workspace_bytes(M, F, K, 1 | (act & (GVQ_SLOPES_ROUNDED | GVQ_SLOPES_PRECISE)), plain);
            if (bytes < 0) return false;
            const at::Tensor ws = room(bytes, c.device);
            return entry.gated_backward(c.h, dh.p, dh.ld, g.p, g.ld, u.p, u.ld, x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld, dh.dtype, M, F, K, act, dx.p, dx.ld,
                                        dg.p, dg.ld, du.p, du.ld, want_g ? dg.dtype : du.dtype, ws.data_ptr(), (size_t)bytes) == GVQ_OK;
        });
    });
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<bind>("bind"),           method<i8_fill>("i8_fill"),             method<i8_quantize>("i8_quantize"),
                         method<i8_matmul>("i8_matmul"), method<i8_gated>("i8_gated"),           method<gated_forward>("gated_forward"),
                         method<gated_backward>("gated_backward"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
