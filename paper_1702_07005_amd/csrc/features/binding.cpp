// binding.cpp -- the Python binding of the operators of learned features: checks a call's tensors, allocates its
// outputs and scratch from torch's allocator, and calls the C entry of include/scd.h.  It is compiled, unlike
// the solver's ctypes binding, because these calls take microseconds: one with two outputs and a workspace
// costs the host 17 us through ctypes and torch's Python functions, of which the two launches are 6.
//
// Every function takes the number of the current device and its current stream first, and returns None where the tensors
// are on another device (paper_1702_07005_amd/features.py then makes that one current and calls again).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/Allocator.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <algorithm>
#include <string>
#include <vector>

#include "scd.h"

namespace {

// Refusals of the binding become ValueError, the C entries' status ScdError.
[[noreturn]] void refuse(const std::string& what) {
    PyErr_SetString(PyExc_ValueError, what.c_str());
    throw python_error();
}

void check(int code) {
    if (code == SCD_OK) return;
    const std::string message = scd_last_error();
    THPObjectPtr module(PyImport_ImportModule("paper_1702_07005_amd.scd"));
    THPObjectPtr type(module ? PyObject_GetAttrString(module, "ScdError") : nullptr);
    THPObjectPtr error(type ? PyObject_CallFunction(type, "is", code, message.c_str()) : nullptr);
    if (error) PyErr_SetObject(type, error);
    throw python_error();
}

// What every call begins with.
struct Call {
    PyObject* const* args;
    int64_t device;
    void* stream;

    Call(PyObject* const* a, Py_ssize_t n, Py_ssize_t want) : args(a + 2) {
        if (n != want + 2) refuse("wrong number of arguments");
        device = number(a[0]);
        stream = reinterpret_cast<void*>(number(a[1]));
    }
    static int64_t number(PyObject* o) {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) throw python_error();
        return v;
    }
    static float real(PyObject* o) {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) throw python_error();
        return (float)v;
    }
    // The k-th argument: a tensor, which lives as long as the call.
    const at::Tensor& tensor(int k, const char* what) const {
        if (!THPVariable_Check(args[k])) refuse(std::string(what) + " must be a tensor");
        return THPVariable_Unpack(args[k]);
    }
    bool given(int k) const { return args[k] != Py_None; }
    bool here(const at::Tensor& t) const { return t.device().index() == device; }
};

int32_t element(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return SCD_F32;
        case at::kBFloat16: return SCD_BF16;
        case at::kHalf: return SCD_F16;
        default: return -1;
    }
}

// A tensor of at least one dimension as rows of its last one.
struct Rows {
    void* data;
    int64_t n, dim, stride;
    int32_t type;
};

Rows rows_of(const at::Tensor& t, const char* what) {
    const int32_t type = element(t.scalar_type());
    const int64_t d = t.dim();
    if (type < 0 || !t.is_cuda() || d < 1)
        refuse(std::string(what) + " must be a CUDA tensor of float32, bfloat16 or float16 with at least one dimension");
    const auto sizes = t.sizes(), strides = t.strides();
    Rows r{t.data_ptr(), 1, sizes[d - 1], sizes[d - 1], type};
    for (int64_t i = 0; i < d - 1; ++i) r.n *= sizes[i];
    if (r.n == 0 || r.dim == 0) return r;
    if (r.dim > 1 && strides[d - 1] != 1) refuse(std::string(what) + ": its last dimension must have unit stride");
    // The leading dimensions have one stride together: each one's step is the next one's length.
    bool first = true;
    int64_t next = 0;
    for (int64_t i = d - 2; i >= 0; --i) {
        if (sizes[i] == 1) continue;
        if (first)
            r.stride = strides[i];
        else if (strides[i] != next)
            refuse(std::string(what) + ": its leading dimensions must have one stride together");
        next = strides[i] * sizes[i];
        first = false;
    }
    return r;
}

const void* vector_of(const at::Tensor& t, const char* what, at::ScalarType type, int64_t n, const at::Device& device) {
    if (t.scalar_type() != type || t.numel() != n || t.device() != device || !t.is_contiguous())
        refuse(std::string(what) + " must be a contiguous tensor with " + std::to_string(n) + " elements of the type " + c10::toString(type) +
               " on the other tensors' device");
    return t.data_ptr();
}

int32_t token_type(const at::Tensor& tokens, const at::Device& device) {
    const at::ScalarType s = tokens.scalar_type();
    if ((s != at::kInt && s != at::kLong) || tokens.device() != device || !tokens.is_contiguous())
        refuse("tokens must be a contiguous int32 or int64 tensor on the other tensors' device");
    return s == at::kInt ? SCD_I32 : SCD_I64;
}

at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Device& device) {
    return at::empty(sizes, at::TensorOptions().dtype(type).device(device));
}

// The calls are outside autograd: they record nothing.  A caller's tensor that they write to counts the write, as
// after an in-place operation of torch, so that autograd notices where it had saved the former values; and one whose own
// history would no longer hold is refused.
void check_writable(const at::Tensor& t, const std::string& what) {
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse(what + " requires gradients, which writing to it would make wrong: call under torch.no_grad(), or detach it");
}

void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The output of a call: `out` if given, else a new tensor of `type`.
struct Output {
    at::Tensor t;
    Rows rows;
    bool given;
    void done() const {
        if (given) written(t);
    }
};

Output output(const Call& c, int out, at::IntArrayRef sizes, at::ScalarType type, const at::Device& device) {
    Output o;
    o.given = c.given(out);
    if (o.given) {
        o.t = c.tensor(out, "out");
        check_writable(o.t, "out");
        if (o.t.sizes() != sizes || o.t.scalar_type() != type || o.t.device() != device)
            refuse(std::string("out must have the result's shape and device and the type ") + c10::toString(type));
    } else {
        o.t = fresh(sizes, type, device);
    }
    o.rows = rows_of(o.t, "out");
    return o;
}

// The type of a result: asked for, that of the output given, or `usual`.
at::ScalarType result_type(const Call& c, int dtype, int out, at::ScalarType usual) {
    at::ScalarType t = usual;
    if (c.given(dtype)) {
        if (!THPDtype_Check(c.args[dtype])) refuse("dtype must be a torch.dtype");
        t = reinterpret_cast<THPDtype*>(c.args[dtype])->scalar_type;
    } else if (c.given(out)) {
        t = c.tensor(out, "out").scalar_type();
    }
    if (element(t) < 0) refuse("dtype must be float32, bfloat16 or float16");
    return t;
}

// Scratch from torch's allocator; it goes back to it at the end of the call, for work that follows on the stream.
struct Scratch {
    c10::DataPtr data;
    int64_t bytes;
    explicit Scratch(int64_t b) : bytes(b) {
        if (b > 0) data = c10::GetAllocator(c10::DeviceType::CUDA)->allocate((size_t)b);
    }
};

std::vector<int64_t> shape_of(at::IntArrayRef lead, int64_t dim) {
    std::vector<int64_t> s(lead.begin(), lead.end());
    s.push_back(dim);
    return s;
}

PyObject* none() { Py_RETURN_NONE; }

// embed(device, stream, tokens, table, scale, out, dtype)
PyObject* embed(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 5);
    const at::Tensor &tokens = c.tensor(0, "tokens"), &table = c.tensor(1, "table");
    const Rows t = rows_of(table, "table");
    if (table.dim() != 2) refuse("table must have two dimensions");
    const int32_t ids = token_type(tokens, table.device());
    if (!c.here(table)) return none();
    const Output o = output(c, 3, shape_of(tokens.sizes(), t.dim), result_type(c, 4, 3, table.scalar_type()), table.device());
    check(scd_embed(tokens.data_ptr(), ids, tokens.numel(), t.data, t.type, t.stride, table.size(0), t.dim, Call::real(c.args[2]),
                    o.rows.data, o.rows.type, o.rows.stride, c.stream));
    o.done();
    return THPVariable_Wrap(o.t);
    END_HANDLE_TH_ERRORS
}

// embed_grad(device, stream, tokens, grad, rows, scale, out, accumulate, dtype)
PyObject* embed_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 7);
    const at::Tensor &tokens = c.tensor(0, "tokens"), &grad = c.tensor(1, "grad");
    const Rows g = rows_of(grad, "grad");
    const int32_t ids = token_type(tokens, grad.device());
    if (grad.sizes().slice(0, grad.dim() - 1) != tokens.sizes()) refuse("grad must have the tokens' shape and one dimension more");
    if (!c.here(grad)) return none();
    const int64_t rows = Call::number(c.args[2]);
    const int accumulate = PyObject_IsTrue(c.args[5]);
    if (accumulate < 0) throw python_error();
    if (accumulate && !c.given(4)) refuse("accumulate needs out");
    int64_t need = 0;
    check(scd_embed_grad_workspace(g.n, rows, g.dim, &need));
    const Output o = output(c, 4, {rows, g.dim}, result_type(c, 6, 4, grad.scalar_type()), grad.device());
    const Scratch work(need);
    check(scd_embed_grad(tokens.data_ptr(), ids, g.n, g.data, g.type, g.stride, rows, g.dim, Call::real(c.args[3]), accumulate,
                         o.rows.data, o.rows.type, o.rows.stride, work.data.get(), need, c.stream));
    o.done();
    return THPVariable_Wrap(o.t);
    END_HANDLE_TH_ERRORS
}

// layer_norm(device, stream, x, weight, bias, eps, out)
PyObject* layer_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 5);
    const at::Tensor& x = c.tensor(0, "x");
    const Rows r = rows_of(x, "x");
    const at::Device device = x.device();
    const at::ScalarType param = c.given(1) ? c.tensor(1, "weight").scalar_type() : c.given(2) ? c.tensor(2, "bias").scalar_type() : x.scalar_type();
    const void* const w = c.given(1) ? vector_of(c.tensor(1, "weight"), "weight", param, r.dim, device) : nullptr;
    const void* const b = c.given(2) ? vector_of(c.tensor(2, "bias"), "bias", param, r.dim, device) : nullptr;
    if (!c.here(x)) return none();
    const Output o = output(c, 4, x.sizes(), x.scalar_type(), device);
    const auto lead = x.sizes().slice(0, x.dim() - 1);
    const at::Tensor mean = fresh(lead, at::kFloat, device), rstd = fresh(lead, at::kFloat, device);
    check(scd_layer_norm(r.data, r.type, r.stride, r.n, r.dim, w, b, element(param), Call::real(c.args[3]), o.rows.data, o.rows.stride,
                         static_cast<float*>(mean.data_ptr()), static_cast<float*>(rstd.data_ptr()), c.stream));
    o.done();
    return Py_BuildValue("(NNN)", THPVariable_Wrap(o.t), THPVariable_Wrap(mean), THPVariable_Wrap(rstd));
    END_HANDLE_TH_ERRORS
}

// layer_norm_grad(device, stream, grad, x, mean, rstd, weight, params, out)
PyObject* layer_norm_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 7);
    const at::Tensor &grad = c.tensor(0, "grad"), &x = c.tensor(1, "x");
    const Rows r = rows_of(x, "x"), g = rows_of(grad, "grad");
    const at::Device device = x.device();
    if (grad.scalar_type() != x.scalar_type() || grad.sizes() != x.sizes() || grad.device() != device) refuse("grad must have x's type, shape and device");
    const void* const m = vector_of(c.tensor(2, "mean"), "mean", at::kFloat, r.n, device);
    const void* const s = vector_of(c.tensor(3, "rstd"), "rstd", at::kFloat, r.n, device);
    const at::ScalarType param = c.given(4) ? c.tensor(4, "weight").scalar_type() : x.scalar_type();
    const void* const w = c.given(4) ? vector_of(c.tensor(4, "weight"), "weight", param, r.dim, device) : nullptr;
    const int params = PyObject_IsTrue(c.args[5]);
    if (params < 0) throw python_error();
    if (!c.here(x)) return none();
    const Output o = output(c, 6, x.sizes(), x.scalar_type(), device);
    at::Tensor dw, db;
    int64_t need = 0;
    if (params) {
        check(scd_layer_norm_grad_workspace(r.n, r.dim, &need));
        dw = fresh({r.dim}, param, device);
        db = fresh({r.dim}, param, device);
    }
    const Scratch work(need);
    check(scd_layer_norm_grad(g.data, g.stride, r.data, r.stride, r.type, static_cast<const float*>(m), static_cast<const float*>(s), r.n, r.dim, w,
                              element(param), o.rows.data, o.rows.stride, params ? dw.data_ptr() : nullptr, params ? db.data_ptr() : nullptr,
                              work.data.get(), need, c.stream));
    o.done();
    if (!params) return Py_BuildValue("(NOO)", THPVariable_Wrap(o.t), Py_None, Py_None);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(o.t), THPVariable_Wrap(dw), THPVariable_Wrap(db));
    END_HANDLE_TH_ERRORS
}

// Refuses a tensor that is written to and shares memory with another one of the call, whose elements would be scaled twice
// or read after the write.  A span that is clipped in place is one range.
void check_apart(const std::vector<scd_span_t>& spans) {
    struct Range {
        uintptr_t from, to;
        bool written;
    };
    const auto bytes = [](int64_t n, int32_t type) { return (uintptr_t)n * (type == SCD_F32 ? 4 : 2); };
    std::vector<Range> ranges;
    ranges.reserve(2 * spans.size());
    bool writes = false;
    for (const scd_span_t& s : spans) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(s.src), q = reinterpret_cast<uintptr_t>(s.dst);
        if (s.n == 0) continue;
        if (p != q) ranges.push_back(Range{p, p + bytes(s.n, s.src_type), false});
        if (q) ranges.push_back(Range{q, q + bytes(s.n, s.dst_type), true});
        writes |= q != 0;
    }
    if (!writes || ranges.size() < 2) return;
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t read = 0, written = 0;  // where the ranges before end
    for (const Range& r : ranges) {
        if (r.from < written || (r.written && r.from < read)) refuse("a tensor that is written to shares memory with another one of the call");
        (r.written ? written : read) = std::max(r.written ? written : read, r.to);
    }
}

// clip(device, stream, grads, outs, max_norm): outs is grads for clipping in place, None for the norm alone.
PyObject* clip(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 3);
    const bool in_place = c.args[1] == c.args[0], norm_only = !c.given(1);
    THPObjectPtr grads(PySequence_Fast(c.args[0], "grads must be a sequence of tensors"));
    if (!grads) throw python_error();
    THPObjectPtr outs(in_place || norm_only ? nullptr : PySequence_Fast(c.args[1], "out must be a sequence of tensors"));
    if (!outs && !in_place && !norm_only) throw python_error();
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(grads.get());
    if (count == 0) refuse("no gradients");
    if (outs && PySequence_Fast_GET_SIZE(outs.get()) != count) refuse("out must have as many tensors as grads");
    std::vector<scd_span_t> spans((size_t)count);
    at::Device device(at::kCPU);
    for (Py_ssize_t i = 0; i < count; ++i) {
        PyObject* const p = PySequence_Fast_GET_ITEM(grads.get(), i);
        if (!THPVariable_Check(p)) refuse("grads must be tensors");
        const at::Tensor& g = THPVariable_Unpack(p);
        if (i == 0) device = g.device();
        const int32_t type = element(g.scalar_type());
        if (type < 0 || !g.is_cuda() || g.device() != device || !g.is_contiguous())
            refuse("gradient " + std::to_string(i) + " must be a contiguous float32, bfloat16 or float16 tensor on the first one's GPU");
        scd_span_t& s = spans[(size_t)i];
        s = scd_span_t{g.data_ptr(), in_place ? g.data_ptr() : nullptr, g.numel(), type, type};
        if (in_place) check_writable(g, "gradient " + std::to_string(i));
        if (!outs) continue;
        PyObject* const q = PySequence_Fast_GET_ITEM(outs.get(), i);
        if (!THPVariable_Check(q)) refuse("out must be tensors");
        const at::Tensor& o = THPVariable_Unpack(q);
        s.dst_type = element(o.scalar_type());
        if ((s.dst_type != type && s.dst_type != SCD_F32) || o.device() != device || o.sizes() != g.sizes() || !o.is_contiguous())
            refuse("output " + std::to_string(i) + " must be contiguous, with its gradient's shape and device, and its type or float32");
        check_writable(o, "output " + std::to_string(i));
        s.dst = o.data_ptr();
    }
    check_apart(spans);
    if (device.index() != c.device) return none();
    int64_t need = 0;
    check(scd_clip_grads_workspace(&need));
    const at::Tensor norm = fresh({}, at::kFloat, device);
    const Scratch work(need);
    check(scd_clip_grads(spans.data(), count, Call::real(c.args[2]), static_cast<float*>(norm.data_ptr()), work.data.get(), need, c.stream));
    if (in_place || outs)
        for (Py_ssize_t i = 0; i < count; ++i) written(THPVariable_Unpack(PySequence_Fast_GET_ITEM((in_place ? grads : outs).get(), i)));
    return THPVariable_Wrap(norm);
    END_HANDLE_TH_ERRORS
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(embed), ENTRY(embed_grad), ENTRY(layer_norm), ENTRY(layer_norm_grad), ENTRY(clip), {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_features", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__features() { return PyModule_Create(&module); }
