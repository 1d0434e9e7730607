// The operators' calls from Python without ctypes and its marshalling: a call on small tensors is host time before anything else (one frame of one sequence 10.4 us
// through ctypes, 4.2 here).  Every function here checks its arguments, allocates the outputs, calls the C ABI and hands the outputs over; where anything is not as it has to
// be it returns None and has done nothing, and operators.py, which knows the same rules, says what is wrong.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sr_rollout.h"

namespace {

// The tensor behind an argument; null where there is none.
const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// Tensors on the current device that no gradient is recorded for, in either direction.
struct Device {
    int index = -1;
    bool fits(const at::Tensor* t)
    {
        if (!t || !t->defined() || !t->is_cuda() || t->layout() != at::kStrided || (c10::GradMode::is_enabled() && t->requires_grad()) ||
            t->_fw_grad(0).defined())
            return false;
        if (index < 0) index = (int)t->get_device();
        return t->get_device() == index;
    }
    bool current() const { return (int)c10::cuda::current_device() == index; }
    void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream(); }
};

// SR_DTYPE_* of a tensor; -1: none
int type_of(const at::Tensor& t)
{
    const auto s = t.scalar_type();
    return s == at::kFloat ? SR_DTYPE_F32 : s == at::kBFloat16 ? SR_DTYPE_BF16 : -1;
}
// A matrix whose rows have no gaps inside.
bool rows_of(const at::Tensor& t, int64_t& stride)
{
    if (t.dim() != 2 || type_of(t) < 0 || t.size(1) < 1 || (t.stride(1) != 1 && t.size(1) > 1)) return false;
    stride = t.size(0) > 1 ? t.stride(0) : t.size(1);
    return true;
}
bool floats(const at::Tensor* t, int64_t n) { return t->scalar_type() == at::kFloat && t->dim() == 1 && t->size(0) == n && t->is_contiguous(); }

// Whether a microscaled matrix's buffers have the sizes that its rows, columns and format make.
bool scaled_fits(const at::Tensor* data, const at::Tensor* scales, int64_t rows, int64_t cols, int format)
{
    size_t data_bytes = 0, scale_bytes = 0;
    return sr_microscale_bytes(rows, cols, format, &data_bytes, &scale_bytes) == SR_OK && data->scalar_type() == at::kByte && scales->scalar_type() == at::kByte &&
           data->is_contiguous() && scales->is_contiguous() && (size_t)data->numel() == data_bytes && (size_t)scales->numel() == scale_bytes;
}

// What was written in place: whoever has kept the tensor for a gradient learns of it.  (Tensors of inference mode have no versions.)
void written(const at::Tensor& t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

PyObject* none() { Py_RETURN_NONE; }
// Without the interpreter's lock: an allocation or a launch may have to wait for the device, which may wait for another thread's launch.
struct Unlocked {
    PyThreadState* const state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};
PyObject* two(PyObject* a, PyObject* b)
{
    PyObject* r = a && b ? PyTuple_New(2) : nullptr;
    if (!r) {
        Py_XDECREF(a);
        Py_XDECREF(b);
        return nullptr;
    }
    PyTuple_SET_ITEM(r, 0, a);
    PyTuple_SET_ITEM(r, 1, b);
    return r;
}
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

// A tensor without values on x's device, by the allocator's own entry (through the dispatcher each costs most of a microsecond more).
at::Tensor new_tensor(const at::Tensor& x, at::IntArrayRef sizes, at::ScalarType type) { return at::Tensor(at::detail::empty_cuda(sizes, type, x.device(), std::nullopt)); }

struct Scaled {
    at::Tensor data, scales;
};
Scaled new_scaled(const at::Tensor& like, int64_t rows, int64_t cols, int format)
{
    const int64_t groups = (cols + 31) / 32;
    return {new_tensor(like, {rows, groups * (format == SR_FORMAT_MX4 ? 16 : 32)}, at::kByte), new_tensor(like, {(rows + 127) / 128 * ((groups + 3) / 4) * 512}, at::kByte)};
}

// No exception of the allocator's leaves through a C function: None, and operators.py meets it again.
#define SR_GUARDED(...)                   \
    try {                                 \
        return [&]() -> PyObject* __VA_ARGS__(); \
    } catch (const std::exception&) {     \
        PyErr_Clear();                    \
        return none();                    \
    }

// quantize(x, format) -> (data, scales)
PyObject* py_quantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 2) return none();
    SR_GUARDED({
        const at::Tensor* x = tensor(a[0]);
        const int format = (int)PyLong_AsLong(a[1]);
        Device d;
        int64_t stride;
        if (!d.fits(x) || !d.current() || !rows_of(*x, stride)) return none();
        Scaled m;
        sr_status st;
        {
            Unlocked u;
            m = new_scaled(*x, x->size(0), x->size(1), format);
            st = sr_microscale_quantize(x->data_ptr(), type_of(*x), x->size(0), x->size(1), stride, format, m.data.data_ptr(), m.scales.data_ptr(), d.stream());
        }
        if (st != SR_OK) return none();
        return two(wrap(m.data), wrap(m.scales));
    })
}

// product(a data, a scales, a rows, w data, w scales, w rows, cols, format, bias or None, relu, dtype, out or None) -> out
PyObject* py_product(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 12) return none();
    SR_GUARDED({
        const at::Tensor *ad = tensor(a[0]), *as = tensor(a[1]), *wd = tensor(a[3]), *ws = tensor(a[4]);
        const int64_t rows = PyLong_AsLongLong(a[2]), outs = PyLong_AsLongLong(a[5]), cols = PyLong_AsLongLong(a[6]);
        const int format = (int)PyLong_AsLong(a[7]), relu = PyObject_IsTrue(a[9]), dtype = (int)PyLong_AsLong(a[10]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return none();
        }
        const at::Tensor *bias = a[8] == Py_None ? nullptr : tensor(a[8]), *given = a[11] == Py_None ? nullptr : tensor(a[11]);
        Device d;
        if (!d.fits(ad) || !d.fits(as) || !d.fits(wd) || !d.fits(ws) || !d.current()) return none();
        if (!scaled_fits(ad, as, rows, cols, format) || !scaled_fits(wd, ws, outs, cols, format)) return none();
        if (a[8] != Py_None && (!d.fits(bias) || !floats(bias, outs))) return none();
        at::Tensor out;
        int64_t stride = outs;
        if (a[11] != Py_None) {
            if (!d.fits(given) || outs < 1 || !rows_of(*given, stride) || given->size(0) != rows || given->size(1) != outs) return none();
            out = *given;
        }
        sr_status st;
        {
            Unlocked u;
            if (!given) out = new_tensor(*ad, {rows, outs}, dtype == SR_DTYPE_F32 ? at::kFloat : at::kBFloat16);
            st = sr_microscale_product(ad->data_ptr(), as->data_ptr(), wd->data_ptr(), ws->data_ptr(), format, rows, cols, outs,
                                       bias ? static_cast<const float*>(bias->data_ptr()) : nullptr, relu ? 1 : 0, out.data_ptr(), type_of(out), stride, d.stream());
        }
        if (st != SR_OK) return none();
        if (given) written(*given);
        return wrap(out);
    })
}

// rms_norm(x, weight or None, residual or None, eps, format or 0) -> (out, or data and scales; sum or None)
PyObject* py_norm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 5) return none();
    SR_GUARDED({
        const at::Tensor *x = tensor(a[0]), *w = a[1] == Py_None ? nullptr : tensor(a[1]), *r = a[2] == Py_None ? nullptr : tensor(a[2]);
        const double eps = PyFloat_AsDouble(a[3]);
        const int format = (int)PyLong_AsLong(a[4]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return none();
        }
        Device d;
        int64_t xs;
        int64_t rs = 0;
        if (!d.fits(x) || !d.current() || !rows_of(*x, xs)) return none();
        const int64_t rows = x->size(0), cols = x->size(1);
        if (a[1] != Py_None && (!d.fits(w) || !floats(w, cols))) return none();
        if (a[2] != Py_None && (!d.fits(r) || !rows_of(*r, rs) || r->size(0) != rows || r->size(1) != cols || r->scalar_type() != x->scalar_type())) return none();
        at::Tensor sum, out;
        Scaled m;
        sr_status st;
        {
            Unlocked u;
            if (r) sum = new_tensor(*x, {rows, cols}, x->scalar_type());
            if (format) m = new_scaled(*x, rows, cols, format);
            else out = new_tensor(*x, {rows, cols}, x->scalar_type());
            st = sr_rms_norm(x->data_ptr(), r ? r->data_ptr() : nullptr, w ? static_cast<const float*>(w->data_ptr()) : nullptr, (float)eps, type_of(*x), rows, cols, xs, rs,
                             r ? sum.data_ptr() : nullptr, format ? m.data.data_ptr() : out.data_ptr(), format ? format : type_of(*x),
                             format ? m.scales.data_ptr() : nullptr, d.stream());
        }
        if (st != SR_OK) return none();
        PyObject* first = format ? two(wrap(m.data), wrap(m.scales)) : wrap(out);
        PyObject* second = r ? wrap(sum) : none();
        return two(first, second);
    })
}

// What run and step have in common; lead: dimensions ahead of the heads.
bool describe(sr_attention_desc& d, Device& dev, const at::Tensor* q, const at::Tensor* k, const at::Tensor* v, const at::Tensor* decay, int lead, bool step, double scale)
{
    if (!dev.fits(q) || !dev.fits(k) || !dev.fits(v) || !dev.fits(decay) || !dev.current()) return false;
    const int type = type_of(*q), dims = lead + 2;
    if (type < 0 || type_of(*k) != type || type_of(*v) != type || decay->scalar_type() != at::kFloat || q->dim() != dims || k->dim() != dims || v->dim() != dims)
        return false;
    for (int i = 0; i < lead; ++i)
        if (k->size(i) != q->size(i) || v->size(i) != q->size(i)) return false;
    const int64_t heads = q->size(lead), groups = k->size(lead), dk = q->size(lead + 1), dv = v->size(lead + 1);
    if (k->size(lead + 1) != dk || v->size(lead) != groups || groups < 1 || heads < 1 || heads % groups || dk < 1 || dv < 1 || heads > 0x7FFFFFFF || dv > 0x7FFFFFFF ||
        dk > 0x7FFFFFFF)
        return false;
    for (const at::Tensor* t : {q, k, v})
        if (t->stride(lead + 1) != 1 && t->size(lead + 1) > 1) return false;
    const bool one = decay->dim() == 1;
    if (one ? decay->size(0) != groups : decay->dim() != lead + 1 || decay->size(lead) != groups) return false;
    for (int i = 0; !one && i < lead; ++i)
        if (decay->size(i) != q->size(i)) return false;
    auto strides = [&](const at::Tensor& t) {
        sr_attention_strides s{0, 0, 0};
        if (step) s.sequence = t.stride(0);
        else s.frame = t.stride(0);
        if (lead == 2) s.sequence = t.stride(1);
        s.head = t.stride(lead);
        return s;
    };
    d.dtype = type;
    d.heads = (int32_t)heads;
    d.groups = (int32_t)groups;
    d.dk = (int32_t)dk;
    d.dv = (int32_t)dv;
    d.frames = step ? 1 : q->size(0);
    d.scale = (float)scale;
    d.q = strides(*q);
    d.k = strides(*k);
    d.v = strides(*v);
    d.log_decay = one ? sr_attention_strides{0, 0, decay->stride(0)} : strides(*decay);
    return true;
}
bool state_fits(Device& dev, const at::Tensor* t, const sr_attention_desc& d)
{
    return dev.fits(t) && t->scalar_type() == at::kFloat && t->dim() == 4 && t->size(0) == d.batch && t->size(1) == d.groups && t->size(2) == d.dk && t->size(3) == d.dv &&
           t->is_contiguous();
}

// step(q, k, v, log_decay, state, scale) -> out
PyObject* py_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 6) return none();
    SR_GUARDED({
        const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]), *decay = tensor(a[3]), *state = tensor(a[4]);
        const double scale = PyFloat_AsDouble(a[5]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return none();
        }
        sr_attention_desc d{};
        Device dev;
        if (!describe(d, dev, q, k, v, decay, 1, true, scale) || q->size(0) > 0x7FFFFFFF) return none();
        d.batch = (int32_t)q->size(0);
        if (!state_fits(dev, state, d)) return none();
        d.out = {0, (int64_t)d.heads * d.dv, d.dv};
        at::Tensor out;
        sr_status st;
        {
            Unlocked u;
            out = new_tensor(*q, {d.batch, d.heads, d.dv}, q->scalar_type());
            st = sr_linear_attention_step(&d, q->data_ptr(), k->data_ptr(), v->data_ptr(), static_cast<const float*>(decay->data_ptr()),
                                          static_cast<float*>(state->data_ptr()), out.data_ptr(), dev.stream());
        }
        if (st != SR_OK) return none();
        written(*state);
        return wrap(out);
    })
}

// run(q, k, v, log_decay, state or None, offsets or None, scale, out or None, state_out or None) -> (out, last)
PyObject* py_run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 9) return none();
    SR_GUARDED({
        const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]), *decay = tensor(a[3]);
        const at::Tensor *state = a[4] == Py_None ? nullptr : tensor(a[4]), *offsets = a[5] == Py_None ? nullptr : tensor(a[5]);
        const at::Tensor *given = a[7] == Py_None ? nullptr : tensor(a[7]), *to = a[8] == Py_None ? nullptr : tensor(a[8]);
        const double scale = PyFloat_AsDouble(a[6]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return none();
        }
        sr_attention_desc d{};
        Device dev;
        const bool packed = a[5] != Py_None;
        if (!describe(d, dev, q, k, v, decay, packed ? 1 : 2, false, scale)) return none();
        if (packed && (!dev.fits(offsets) || offsets->scalar_type() != at::kLong || offsets->dim() != 1 || offsets->size(0) < 1 || !offsets->is_contiguous())) return none();
        const int64_t batch = packed ? offsets->size(0) - 1 : q->size(1);
        if (batch > 0x7FFFFFFF) return none();
        d.batch = (int32_t)batch;
        if (a[4] != Py_None && !state_fits(dev, state, d)) return none();
        if (a[8] != Py_None && !state_fits(dev, to, d)) return none();
        const int64_t row = (int64_t)d.heads * d.dv;
        d.out = packed ? sr_attention_strides{row, 0, d.dv} : sr_attention_strides{row * batch, row, d.dv};
        at::Tensor out;
        if (a[7] != Py_None) {
            if (!dev.fits(given) || given->scalar_type() != q->scalar_type() || !given->is_contiguous() || given->dim() != q->dim()) return none();
            for (int i = 0; i < q->dim(); ++i)
                if (given->size(i) != (i + 1 < q->dim() ? q->size(i) : d.dv)) return none();
            out = *given;
        }
        at::Tensor last = to ? *to : at::Tensor();
        sr_status st;
        {
            Unlocked u;
            if (!given) out = packed ? new_tensor(*q, {q->size(0), d.heads, d.dv}, q->scalar_type()) : new_tensor(*q, {q->size(0), batch, d.heads, d.dv}, q->scalar_type());
            if (!to) last = new_tensor(*q, {batch, d.groups, d.dk, d.dv}, at::kFloat);
            size_t bytes = 0;
            st = sr_linear_attention_workspace_bytes(&d, packed ? 1 : 0, &bytes);
            at::Tensor work;
            if (st == SR_OK && bytes) work = new_tensor(*q, {(int64_t)bytes}, at::kByte);
            if (st == SR_OK)
                st = sr_linear_attention_run(&d, q->data_ptr(), k->data_ptr(), v->data_ptr(), static_cast<const float*>(decay->data_ptr()),
                                             packed ? static_cast<const int64_t*>(offsets->data_ptr()) : nullptr, state ? static_cast<const float*>(state->data_ptr()) : nullptr,
                                             static_cast<float*>(last.data_ptr()), out.data_ptr(), bytes ? work.data_ptr() : nullptr, bytes, dev.stream());
        }
        if (st != SR_OK) return none();
        if (given) written(*given);
        if (to) written(*to);
        return two(wrap(out), wrap(last));
    })
}

PyMethodDef methods[] = {
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_quantize)), METH_FASTCALL, nullptr},
    {"product", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_product)), METH_FASTCALL, nullptr},
    {"rms_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_norm)), METH_FASTCALL, nullptr},
    {"step", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_step)), METH_FASTCALL, nullptr},
    {"run", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_run)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_operators", "Fast path of operators.py.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&module); }
