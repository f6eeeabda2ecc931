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
#include <ATen/hip/EmptyTensor.h>
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
    static double real64(PyObject* o) {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) throw python_error();
        return v;
    }
    static float real(PyObject* o) { return (float)real64(o); }
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

// `eight`: of 8 bits (e4m3).
Rows rows_of(const at::Tensor& t, const char* what, bool eight = false) {
    const int32_t type = eight ? t.scalar_type() == at::kFloat8_e4m3fn ? SCD_E4M3 : -1 : element(t.scalar_type());
    const int64_t d = t.dim();
    if (type < 0 || !t.is_cuda() || d < 1)
        refuse(std::string(what) + " must be a CUDA tensor of " + (eight ? "float8_e4m3fn" : "float32, bfloat16 or float16") + " with at least one dimension");
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

// What at::empty makes, without its way through the dispatcher.
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Device& device) {
    return at::detail::empty_cuda(sizes, type, device, std::nullopt);
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

// A range of memory that a call over many tensors reads or writes.
struct Range {
    uintptr_t from, to;
    bool written;
};

struct Ranges {
    std::vector<Range> all;
    bool writes = false;
    void add(const void* p, int64_t bytes, bool written) {
        const uintptr_t from = reinterpret_cast<uintptr_t>(p);
        if (bytes == 0) return;
        all.push_back(Range{from, from + (uintptr_t)bytes, written});
        writes |= written;
    }
    void add(const at::Tensor& t, bool written) { add(t.data_ptr(), (int64_t)t.nbytes(), written); }
    // Refuses a tensor that is written to and shares memory with another one of the call, whose elements would be written
    // twice or read after the write.
    void check_apart() {
        if (!writes || all.size() < 2) return;
        std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
        uintptr_t read = 0, written = 0;  // where the ranges before end
        for (const Range& r : all) {
            if (r.from < written || (r.written && r.from < read)) refuse("a tensor that is written to shares memory with another one of the call");
            (r.written ? written : read) = std::max(r.written ? written : read, r.to);
        }
    }
};

// A span that is clipped in place is one range.
void check_apart(const std::vector<scd_span_t>& spans) {
    const auto bytes = [](int64_t n, int32_t type) { return n * (type == SCD_F32 ? 4 : 2); };
    Ranges ranges;
    ranges.all.reserve(2 * spans.size());
    for (const scd_span_t& s : spans) {
        if (s.src != s.dst) ranges.add(s.src, bytes(s.n, s.src_type), false);
        if (s.dst) ranges.add(s.dst, bytes(s.n, s.dst_type), true);
    }
    ranges.check_apart();
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

// Whether the rows of a matrix share memory with those of another.  Matrices side by side in one buffer do not.
bool share(const Rows& a, int64_t asize, const Rows& b, int64_t bsize) {
    if (a.n == 0 || a.dim == 0 || b.n == 0 || b.dim == 0) return false;
    const auto end = [](const Rows& r, int64_t size) { return reinterpret_cast<uintptr_t>(r.data) + (uintptr_t)(((r.n - 1) * r.stride + r.dim) * size); };
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.data), pb = reinterpret_cast<uintptr_t>(b.data);
    if (pa >= end(b, bsize) || pb >= end(a, asize)) return false;
    const uintptr_t step = (uintptr_t)(a.stride * asize), wa = (uintptr_t)(a.dim * asize), wb = (uintptr_t)(b.dim * bsize);
    if (a.n < 2 || b.n < 2 || b.stride * bsize != a.stride * asize || wa > step || wb > step) return true;
    const uintptr_t off = pb >= pa ? (pb - pa) % step : step - 1 - (pa - pb - 1) % step;  // of b's rows in a's
    return off < wa || off + wb > step;
}

// Refuses an output that shares memory with an input, unless it takes its place.
void check_place(const Rows& out, int64_t osize, const Rows& in, int64_t isize, const char* what, const char* which) {
    const bool place = out.data == in.data && osize == isize && (out.stride == in.stride || out.n == 1);
    if (!place && share(out, osize, in, isize)) refuse(std::string(what) + " shares memory with " + which + " without taking its place");
}

Rows vector_rows(const void* p, int64_t n) { return Rows{const_cast<void*>(p), p ? 1 : 0, n, n, 0}; }

// A residual or a gradient that goes with x.
Rows like(const at::Tensor& t, const at::Tensor& x, const char* what) {
    if (t.scalar_type() != x.scalar_type() || t.sizes() != x.sizes() || t.device() != x.device()) refuse(std::string(what) + " must have x's type, shape and device");
    return rows_of(t, what);
}

PyObject* wrap_or_none(const at::Tensor& t) {
    if (!t.defined()) return none();
    return THPVariable_Wrap(t);
}

// rms_norm(device, stream, x, weight, residual, eps, out, sum_out, group): group is None for an output of x's type, else the
// columns of a scale of 8 bits, 0 for the row.
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 7);
    const at::Tensor& x = c.tensor(0, "x");
    const Rows r = rows_of(x, "x");
    const at::Device device = x.device();
    const bool eight = c.given(6);
    const int64_t group = eight ? Call::number(c.args[6]) : 0;
    const at::ScalarType param = c.given(1) ? c.tensor(1, "weight").scalar_type() : x.scalar_type();
    const void* const w = c.given(1) ? vector_of(c.tensor(1, "weight"), "weight", param, r.dim, device) : nullptr;
    const Rows res = c.given(2) ? like(c.tensor(2, "residual"), x, "residual") : Rows{nullptr, 0, 0, 0, 0};
    if (c.given(5) && !c.given(2)) refuse("sum_out needs a residual");
    if (!c.here(x)) return none();
    const int64_t size = (int64_t)x.element_size();
    at::Tensor y, scale, sum;
    if (c.given(4)) {
        y = c.tensor(4, "out");
        check_writable(y, "out");
        if (y.sizes() != x.sizes() || y.scalar_type() != (eight ? at::kFloat8_e4m3fn : x.scalar_type()) || y.device() != device)
            refuse(std::string("out must have x's shape and device and the type ") + c10::toString(eight ? at::kFloat8_e4m3fn : x.scalar_type()));
    } else {
        y = fresh(x.sizes(), eight ? at::kFloat8_e4m3fn : x.scalar_type(), device);
    }
    const Rows o = rows_of(y, "out", eight);
    if (c.given(2)) {
        sum = c.given(5) ? c.tensor(5, "sum_out") : fresh(x.sizes(), x.scalar_type(), device);
        if (c.given(5)) check_writable(sum, "sum_out");
    }
    const Rows h = c.given(2) ? like(sum, x, "sum_out") : Rows{nullptr, 0, 0, 0, 0};
    if (c.given(4)) {
        check_place(o, eight ? 1 : size, r, size, "out", "x");
        check_place(o, eight ? 1 : size, res, size, "out", "residual");
        if (share(o, eight ? 1 : size, vector_rows(w, r.dim), w ? (int64_t)c10::elementSize(param) : 1)) refuse("out shares memory with weight");
    }
    if (c.given(5)) {
        check_place(h, size, r, size, "sum_out", "x");
        check_place(h, size, res, size, "sum_out", "residual");
        if (share(h, size, vector_rows(w, r.dim), w ? (int64_t)c10::elementSize(param) : 1)) refuse("sum_out shares memory with weight");
        if (share(o, eight ? 1 : size, h, size)) refuse("out shares memory with sum_out");
    }
    const auto lead = x.sizes().slice(0, x.dim() - 1);
    if (eight) scale = group ? fresh(shape_of(lead, group > 0 ? (r.dim + group - 1) / group : 0), at::kFloat, device) : fresh(lead, at::kFloat, device);
    const at::Tensor rstd = fresh(lead, at::kFloat, device);
    check(scd_rms_norm(r.data, r.type, r.stride, res.data, res.stride, r.n, r.dim, w, element(param), Call::real(c.args[3]), o.data, eight ? SCD_E4M3 : r.type, o.stride,
                       eight ? static_cast<float*>(scale.data_ptr()) : nullptr, group, h.data, h.stride, static_cast<float*>(rstd.data_ptr()), c.stream));
    if (c.given(4)) written(y);
    if (c.given(5)) written(sum);
    // x is h, but not where it holds y now.
    if (!sum.defined() && x.requires_grad()) sum = x.detach();
    PyObject* const kept = o.data == r.data && r.n > 0 && !c.given(2) ? none() : sum.defined() ? THPVariable_Wrap(sum) : Py_NewRef(c.args[0]);
    if (eight) return Py_BuildValue("(NNNN)", THPVariable_Wrap(y), THPVariable_Wrap(scale), THPVariable_Wrap(rstd), kept);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(y), THPVariable_Wrap(rstd), kept);
    END_HANDLE_TH_ERRORS
}

// rms_norm_grad(device, stream, grad, x, rstd, weight, residual_grad, params, out)
PyObject* rms_norm_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 7);
    const at::Tensor &grad = c.tensor(0, "grad"), &x = c.tensor(1, "x");
    const Rows r = rows_of(x, "x"), g = like(grad, x, "grad");
    const at::Device device = x.device();
    const void* const s = vector_of(c.tensor(2, "rstd"), "rstd", at::kFloat, r.n, device);
    const at::ScalarType param = c.given(3) ? c.tensor(3, "weight").scalar_type() : x.scalar_type();
    const void* const w = c.given(3) ? vector_of(c.tensor(3, "weight"), "weight", param, r.dim, device) : nullptr;
    const Rows res = c.given(4) ? like(c.tensor(4, "residual_grad"), x, "residual_grad") : Rows{nullptr, 0, 0, 0, 0};
    const int params = PyObject_IsTrue(c.args[5]);
    if (params < 0) throw python_error();
    if (!c.here(x)) return none();
    const Output o = output(c, 6, x.sizes(), x.scalar_type(), device);
    if (o.given) {
        const int64_t size = (int64_t)x.element_size();
        check_place(o.rows, size, g, size, "out", "grad");
        check_place(o.rows, size, r, size, "out", "x");
        check_place(o.rows, size, res, size, "out", "residual_grad");
        if (share(o.rows, size, vector_rows(s, r.n), 4)) refuse("out shares memory with rstd");
        if (share(o.rows, size, vector_rows(w, r.dim), w ? (int64_t)c10::elementSize(param) : 1)) refuse("out shares memory with weight");
    }
    at::Tensor dw;
    int64_t need = 0;
    if (params) {
        check(scd_rms_norm_grad_workspace(r.n, r.dim, &need));
        dw = fresh({r.dim}, param, device);
    }
    const Scratch work(need);
    check(scd_rms_norm_grad(g.data, g.stride, r.data, r.stride, r.type, static_cast<const float*>(s), r.n, r.dim, w, element(param), res.data, res.stride,
                            o.rows.data, o.rows.stride, params ? dw.data_ptr() : nullptr, work.data.get(), need, c.stream));
    o.done();
    return Py_BuildValue("(NN)", THPVariable_Wrap(o.t), wrap_or_none(dw));
    END_HANDLE_TH_ERRORS
}

// A sequence argument, as a list or tuple.
THPObjectPtr sequence(PyObject* o, const char* what) {
    THPObjectPtr s(PySequence_Fast(o, (std::string(what) + " must be a sequence").c_str()));
    if (!s) throw python_error();
    return s;
}

const at::Tensor& item(PyObject* list, Py_ssize_t i, const char* what) {
    PyObject* const p = PySequence_Fast_GET_ITEM(list, i);
    if (!THPVariable_Check(p)) refuse(std::string(what) + " must be tensors");
    return THPVariable_Unpack(p);
}

// A device scalar of the given type.
const at::Tensor& scalar(const Call& c, int k, const char* what, at::ScalarType type, const at::Device& device) {
    const at::Tensor& t = c.tensor(k, what);
    vector_of(t, what, type, 1, device);
    return t;
}

// adamw(device, stream, params, grads, state, step, lr, beta1, beta2, eps, weight_decay, norm, max_norm, copies, seed): step and
// lr are numbers or device scalars, weight_decay a number or a sequence of them.
PyObject* adamw(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 13);
    THPObjectPtr params = sequence(c.args[0], "params"), grads = sequence(c.args[1], "grads"), states = sequence(c.args[2], "state");
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(params.get());
    if (count == 0) refuse("no parameters");
    if (PySequence_Fast_GET_SIZE(grads.get()) != count || PySequence_Fast_GET_SIZE(states.get()) != count)
        refuse("params, grads and state must have as many entries");
    THPObjectPtr copies, decays;
    if (c.given(11)) {
        copies = sequence(c.args[11], "copies");
        if (PySequence_Fast_GET_SIZE(copies.get()) != count) refuse("copies must have as many entries as params");
    }
    float decay = 0.0f;
    if (PySequence_Check(c.args[8])) {
        decays = sequence(c.args[8], "weight_decay");
        if (PySequence_Fast_GET_SIZE(decays.get()) != count) refuse("weight_decay must have as many entries as params");
    } else {
        decay = Call::real(c.args[8]);
    }
    const at::Device device = item(params.get(), 0, "params").device();
    if (!device.is_cuda()) refuse("params must be CUDA tensors");
    std::vector<scd_adamw_span_t> spans((size_t)count);
    std::vector<const at::Tensor*> writes;
    writes.reserve((size_t)count * 6);
    Ranges ranges;
    ranges.all.reserve((size_t)count * 7 + 3);
    // A tensor of the call that belongs to the i-th parameter.
    const auto take = [&](const at::Tensor& t, const char* what, Py_ssize_t i, at::IntArrayRef sizes, bool write) {
        if (t.device() != device || t.sizes() != sizes || !t.is_contiguous())
            refuse(std::string(what) + " " + std::to_string(i) + " must be contiguous, with its parameter's shape, on the first parameter's GPU");
        if (write) {
            if (t.requires_grad()) check_writable(t, std::string(what) + " " + std::to_string(i));
            writes.push_back(&t);
        }
        ranges.add(t, write);
        return t.data_ptr();
    };
    for (Py_ssize_t i = 0; i < count; ++i) {
        const at::Tensor &p = item(params.get(), i, "params"), &g = item(grads.get(), i, "grads");
        scd_adamw_span_t& s = spans[(size_t)i];
        s = scd_adamw_span_t{};
        const auto sizes = p.sizes();
        s.n = p.numel();
        s.param_type = element(p.scalar_type());
        s.grad_type = element(g.scalar_type());
        if (s.param_type < 0 || s.grad_type < 0) refuse("params and grads must be float32, bfloat16 or float16");
        s.param = take(p, "parameter", i, sizes, true);
        s.grad = take(g, "gradient", i, sizes, false);
        PyObject* const state = PySequence_Fast_GET_ITEM(states.get(), i);
        const Py_ssize_t parts = PyTuple_Check(state) || PyList_Check(state) ? PySequence_Fast_GET_SIZE(state) : 0;
        if (parts != 2 && parts != 4) refuse("an entry of state has two tensors (32 bits) or four (8 bits)");
        const at::ScalarType held = parts == 2 ? at::kFloat : at::kFloat8_e4m3fn;
        const at::Tensor &m = item(state, 0, "states"), &v = item(state, 1, "states");
        if (m.scalar_type() != held || v.scalar_type() != held) refuse(std::string("state ") + std::to_string(i) + " must be of the type " + c10::toString(held));
        s.m = take(m, "state", i, sizes, true);
        s.v = take(v, "state", i, sizes, true);
        s.state_type = parts == 2 ? SCD_F32 : SCD_E4M3;
        if (parts == 4) {
            const int64_t blocks[1] = {(s.n + 255) / 256};
            const at::Tensor &ms = item(state, 2, "states"), &vs = item(state, 3, "states");
            if (ms.scalar_type() != at::kFloat || vs.scalar_type() != at::kFloat || ms.sizes() != at::IntArrayRef(blocks) || vs.sizes() != at::IntArrayRef(blocks))
                refuse("scales of state " + std::to_string(i) + " must be float32 with one element for each 256 of the parameter");
            s.m_scale = static_cast<float*>(take(ms, "scales of state", i, blocks, true));
            s.v_scale = static_cast<float*>(take(vs, "scales of state", i, blocks, true));
        }
        if (copies && PySequence_Fast_GET_ITEM(copies.get(), i) != Py_None) {
            const at::Tensor& q = item(copies.get(), i, "copies");
            s.copy_type = element(q.scalar_type());
            if (s.param_type != SCD_F32 || (s.copy_type != SCD_BF16 && s.copy_type != SCD_F16)) refuse("copies must be bfloat16 or float16, of float32 parameters");
            s.copy = take(q, "copy", i, sizes, true);
        }
        s.weight_decay = decays ? Call::real(PySequence_Fast_GET_ITEM(decays.get(), i)) : decay;
    }
    scd_adamw_t o{};
    const auto read = [&](const at::Tensor& t) {
        ranges.add(t, false);
        return t.data_ptr();
    };
    if (THPVariable_Check(c.args[3]))
        o.step_dev = static_cast<const int64_t*>(read(scalar(c, 3, "step", at::kLong, device)));
    else
        o.step = Call::number(c.args[3]);
    if (THPVariable_Check(c.args[4]))
        o.lr_dev = static_cast<const float*>(read(scalar(c, 4, "lr", at::kFloat, device)));
    else
        o.lr = Call::real64(c.args[4]);
    if (c.given(9)) o.norm_dev = static_cast<const float*>(read(scalar(c, 9, "norm", at::kFloat, device)));
    o.beta1 = Call::real64(c.args[5]);
    o.beta2 = Call::real64(c.args[6]);
    o.eps = Call::real64(c.args[7]);
    o.max_norm = Call::real(c.args[10]);
    const int64_t seed = Call::number(c.args[12]);
    if (seed < 0 || seed > 0xFFFFFFFFLL) refuse("seed must be in [0, 2^32)");
    o.seed = (uint32_t)seed;
    ranges.check_apart();
    if (device.index() != c.device) return none();
    check(scd_adamw(spans.data(), count, &o, c.stream));
    for (const at::Tensor* t : writes) written(*t);
    return Py_NewRef(Py_True);
    END_HANDLE_TH_ERRORS
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(embed), ENTRY(embed_grad), ENTRY(layer_norm), ENTRY(layer_norm_grad), ENTRY(clip), ENTRY(rms_norm), ENTRY(rms_norm_grad), ENTRY(adamw), {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_features", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__features() { return PyModule_Create(&module); }
