// Argument marshalling of the Python binding for the sequence operators: shapes, types, devices and strides of the tensors are
// checked and put into the C ABI's structs here.  In Python the dozen tensors of a call cost 9 us, more than its kernel; here one
// is looked at through its C++ object, and the call costs 1 to 2 us besides the launch.  Computes nothing.  The interpreter lock is
// released around the call, as in ssam_marshal.c.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/Functions.h>

#include <cmath>
#include <cstring>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/ssam_sequence.h"

namespace {

using at::Tensor;

struct {
    decltype(&ssam_conv1d) conv1d;
    decltype(&ssam_conv1d_backward) conv1d_backward;
    decltype(&ssam_conv1d_backward_workspace_bytes) conv1d_backward_bytes;
    decltype(&ssam_conv1d_step) conv1d_step;
    decltype(&ssam_scan_selective) scan;
    decltype(&ssam_scan_selective_workspace_bytes) scan_bytes;
    decltype(&ssam_scan_selective_marks) scan_marks;
    decltype(&ssam_scan_selective_backward) scan_backward;
    decltype(&ssam_scan_selective_backward_workspace_bytes) scan_backward_bytes;
    decltype(&ssam_scan_selective_step) scan_step;
    decltype(&ssam_scan_delta) delta;
    decltype(&ssam_scan_delta_workspace_bytes) delta_bytes;
    decltype(&ssam_scan_delta_marks) delta_marks;
    decltype(&ssam_scan_delta_step) delta_step;
    decltype(&ssam_rms_norm) norm;
    decltype(&ssam_rms_norm_e4m3) norm_e4m3;
    decltype(&ssam_rms_norm_backward) norm_backward;
    decltype(&ssam_rms_norm_backward_workspace_bytes) norm_backward_bytes;
    decltype(&ssam_scan_delta_backward) delta_backward;
    decltype(&ssam_scan_delta_backward_workspace_bytes) delta_backward_bytes;
} entry;
PyObject* status_error;      // the binding's exception class, called with (status, entry point)

struct Bad : std::runtime_error {          // ValueError
    using std::runtime_error::runtime_error;
};
struct BadType : std::runtime_error {      // TypeError
    using std::runtime_error::runtime_error;
};

[[noreturn]] void fail(const char* name, const std::string& what) { throw Bad(std::string(name) + " " + what); }

std::string shape_text(at::IntArrayRef s)
{
    std::string t = "(";
    for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
    return t + (s.size() == 1 ? ",)" : ")");
}
std::string type_text(at::ScalarType t)
{
    return t == at::kFloat8_e4m3fn ? "torch.float8_e4m3fn" : t == at::kFloat ? "torch.float32" : t == at::kHalf ? "torch.float16" : t == at::kBFloat16 ? "torch.bfloat16" : t == at::kInt ? "torch.int32" : c10::toString(t);
}

const Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) throw BadType(std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}
const Tensor* optional(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

int code_of(at::ScalarType t, const char* name)
{
    if (t == at::kFloat) return SSAM_F32;
    if (t == at::kHalf) return SSAM_F16;
    if (t == at::kBFloat16) return SSAM_BF16;
    throw BadType(std::string(name) + ": unsupported dtype " + type_text(t));
}

// The tensor the others are measured by.
const Tensor& main_rows(PyObject* o, const char* name)
{
    const Tensor& t = tensor(o, name);
    if (!t.is_cuda()) fail(name, "must live in GPU memory");
    if (t.dim() != 2 && t.dim() != 3) fail(name, "must be [rows, channels] or [sequences, rows, channels]");
    return t;
}

void same_kind(const Tensor& t, const char* name, at::ScalarType type, const Tensor& like)
{
    if (t.scalar_type() != type || t.device() != like.device()) fail(name, "must be " + type_text(type) + " on " + like.device().str());
}

// like's element type, device and leading extents, channels contiguous.
ssam_rows rows(const Tensor* t, const char* name, const Tensor& like)
{
    if (!t) return ssam_rows{nullptr, 0, 0};
    if (t->sizes() != like.sizes()) fail(name, "must have shape " + shape_text(like.sizes()) + ", not " + shape_text(t->sizes()));
    same_kind(*t, name, like.scalar_type(), like);
    const auto s = t->strides();
    if (s.back() != 1 && t->sizes().back() != 1) fail(name, "must have contiguous channels (stride 1)");
    return s.size() == 2 ? ssam_rows{t->data_ptr(), 0, s[0]} : ssam_rows{t->data_ptr(), s[0], s[1]};
}

// The same for [.., groups, states].
ssam_rows group_rows(const Tensor& t, const char* name, const Tensor& like, long long* apart)
{
    same_kind(t, name, like.scalar_type(), like);
    const auto lead = like.sizes().slice(0, like.dim() - 1);
    if (t.dim() != like.dim() + 1 || t.sizes().slice(0, lead.size()) != lead)
        fail(name, "must have shape " + shape_text(lead) + " + (groups, states), not " + shape_text(t.sizes()));
    const auto s = t.strides();
    if (s.back() != 1 && t.sizes().back() != 1) fail(name, "must have contiguous states (stride 1)");
    *apart = s[s.size() - 2];
    return s.size() == 3 ? ssam_rows{t.data_ptr(), 0, s[0]} : ssam_rows{t.data_ptr(), s[0], s[1]};
}

template <class P = const void>
P* dense(const Tensor* t, const char* name, const Tensor& like, at::ScalarType type, at::IntArrayRef shape)
{
    if (!t) return nullptr;
    if (t->sizes() != shape) fail(name, "must have shape " + shape_text(shape) + ", not " + shape_text(t->sizes()));
    same_kind(*t, name, type, like);
    if (!t->is_contiguous()) fail(name, "must be contiguous");
    return static_cast<P*>(t->data_ptr());
}

int held_to_int(int64_t v, const char* name)
{
    if (v > (1LL << 30)) fail(name, "is too large");
    return (int)v;
}

// `tail`: dimensions of a row.
ssam_sequences sequences(const Tensor& like, const Tensor* starts, const Tensor* lengths, int tail = 1)
{
    if (starts && lengths) fail("starts", "and lengths exclude one another");
    ssam_sequences q{1, held_to_int(like.size(-1 - tail), "the number of rows"), nullptr, nullptr};
    if (like.dim() == 1 + tail) {
        if (lengths) fail("lengths", "belongs to [sequences, rows, channels]");
        if (!starts) return q;
        if (starts->dim() != 1 || starts->numel() < 1 || !starts->is_contiguous()) fail("starts", "must be a contiguous 1D tensor of sequences + 1 offsets");
        same_kind(*starts, "starts", at::kInt, like);
        q.sequences = held_to_int(starts->numel() - 1, "the number of sequences");
        q.d_begin = static_cast<const int*>(starts->data_ptr());
        q.d_end = q.d_begin + 1;
        return q;
    }
    if (starts) fail("starts", "belongs to packed [rows, channels]");
    q.sequences = held_to_int(like.size(0), "the number of sequences");
    if (!lengths) return q;
    if (lengths->dim() != 1 || lengths->numel() != q.sequences || !lengths->is_contiguous())
        fail("lengths", "must be a contiguous 1D tensor of " + std::to_string(q.sequences) + " lengths");
    same_kind(*lengths, "lengths", at::kInt, like);
    q.d_end = static_cast<const int*>(lengths->data_ptr());
    if (!q.sequences) q.d_end = nullptr;
    return q;
}

// A result passed in, or a new one: zeros where rows may belong to no sequence.
Tensor result(const Tensor* given, const Tensor& like, bool ragged)
{
    if (given) return *given;
    return ragged ? at::zeros(like.sizes(), like.options()) : at::empty(like.sizes(), like.options());
}

Tensor workspace(size_t bytes, const Tensor* given, const Tensor& like)
{
    if (given) {
        if (given->device() != like.device() || !given->is_contiguous()) fail("d_work", "must be contiguous on " + like.device().str());
        return *given;
    }
    return bytes ? at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)) : Tensor();
}

PyObject* wrap(const Tensor& t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

template <class Args>
void call(int (*f)(const Args*, void*), const Args& a, PyObject* stream, const char* name)
{
    void* s = PyLong_AsVoidPtr(stream);
    if (PyErr_Occurred()) throw BadType("the stream must be an integer handle");
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f(&a, s);
    Py_END_ALLOW_THREADS
    if (status == SSAM_OK) return;
    PyObject* e = PyObject_CallFunction(status_error, "is", status, name);
    if (e) {
        PyErr_SetObject(status_error, e);
        Py_DECREF(e);
    }
    throw 0;             // the Python error is set
}

// Runs f with C++ exceptions turned into Python's.
template <class F>
PyObject* guarded(F f)
{
    try {
        return f();
    } catch (int) {
    } catch (const Bad& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const BadType& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const c10::OutOfMemoryError& e) {      // as torch's own functions raise it
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* kind = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (kind) PyErr_SetString(kind, e.what_without_backtrace());
        Py_XDECREF(kind);
        Py_XDECREF(torch);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

bool arity(Py_ssize_t have, Py_ssize_t want)
{
    if (have == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", have, want);
    return false;
}

bool truth(PyObject* o)
{
    const int t = PyObject_IsTrue(o);
    if (t < 0) throw 0;
    return t != 0;
}

// ---- filter ------------------------------------------------------------------------------------------------------------
template <class Args>
void filter(Args* a, const Tensor& x, PyObject* weight, PyObject* bias, PyObject* silu)
{
    const Tensor& w = tensor(weight, "weight");
    a->dtype = code_of(x.scalar_type(), "d_in");
    const int64_t channels = x.size(-1);
    if (w.dim() != 2 || w.size(0) != channels) fail("weight", "must have shape (" + std::to_string(channels) + ", taps), not " + shape_text(w.sizes()));
    if (w.scalar_type() != x.scalar_type() && w.scalar_type() != at::kFloat) fail("weight", "must be " + type_text(x.scalar_type()) + " or torch.float32");
    a->param_dtype = code_of(w.scalar_type(), "weight");
    a->channels = held_to_int(channels, "the number of channels");
    a->taps = held_to_int(w.size(1), "the number of taps");
    a->silu = truth(silu);
    a->d_weight = dense(&w, "weight", x, w.scalar_type(), w.sizes());
    a->d_bias = dense(optional(bias, "bias"), "bias", x, w.scalar_type(), {channels});
}

// conv1d(d_in, weight, bias, silu, d_state, d_final, starts, lengths, d_out, stream) -> d_out
PyObject* conv1d(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 10)) return nullptr;
    return guarded([&] {
        const Tensor& x = main_rows(v[0], "d_in");
        ssam_conv1d_args a{};
        filter(&a, x, v[1], v[2], v[3]);
        a.seq = sequences(x, optional(v[6], "starts"), optional(v[7], "lengths"));
        const int64_t carried[] = {a.seq.sequences, a.taps - 1, a.channels};
        a.d_state = dense(optional(v[4], "d_state"), "d_state", x, x.scalar_type(), carried);
        a.d_final = dense<void>(optional(v[5], "d_final"), "d_final", x, x.scalar_type(), carried);
        const Tensor* given = optional(v[8], "d_out");
        const Tensor out = result(given, x, a.seq.d_begin || a.seq.d_end);
        a.in = rows(&x, "d_in", x);
        a.out = rows(&out, "d_out", x);
        call(entry.conv1d, a, v[9], "ssam_conv1d");
        if (given) {
            Py_INCREF(v[8]);
            return v[8];
        }
        return wrap(out);
    });
}

// conv1d_backward(d_grad, d_in, weight, bias, silu, d_state, d_grad_final, starts, lengths, state_grad, d_work, stream)
//     -> (x, weight, bias, state)
PyObject* conv1d_backward(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 12)) return nullptr;
    return guarded([&] {
        const Tensor& x = main_rows(v[1], "d_in");
        ssam_conv1d_backward_args a{};
        filter(&a, x, v[2], v[3], v[4]);
        a.seq = sequences(x, optional(v[7], "starts"), optional(v[8], "lengths"));
        const int64_t carried[] = {a.seq.sequences, a.taps - 1, a.channels};
        a.d_state = dense(optional(v[5], "d_state"), "d_state", x, x.scalar_type(), carried);
        a.d_grad_final = dense(optional(v[6], "d_grad_final"), "d_grad_final", x, x.scalar_type(), carried);
        a.in = rows(&x, "d_in", x);
        a.grad_out = rows(&tensor(v[0], "d_grad"), "d_grad", x);
        const Tensor& w = tensor(v[2], "weight");
        const Tensor gx = result(nullptr, x, a.seq.d_begin || a.seq.d_end), gw = at::empty(w.sizes(), w.options());
        const Tensor gb = v[3] == Py_None ? Tensor() : at::empty({a.channels}, w.options());
        const Tensor gs = truth(v[9]) ? at::empty(carried, x.options()) : Tensor();
        a.grad_in = rows(&gx, "x", x);
        a.d_grad_weight = gw.data_ptr();
        if (gb.defined()) a.d_grad_bias = gb.data_ptr();
        if (gs.defined()) a.d_grad_state = gs.data_ptr();
        const Tensor work = workspace(entry.conv1d_backward_bytes(&a), optional(v[10], "d_work"), x);
        if (work.defined()) {
            a.d_work = work.data_ptr();
            a.work_bytes = work.nbytes();
        }
        call(entry.conv1d_backward, a, v[11], "ssam_conv1d_backward");
        return Py_BuildValue("(NNNN)", wrap(gx), wrap(gw), wrap(gb), wrap(gs));
    });
}

// Slots of a pool [slots, ..]: each contiguous, `slot` elements, none over another.
void pool(const Tensor& t, at::ScalarType type, const Tensor& like, std::initializer_list<int64_t> shape, long long* stride, int* slots)
{
    std::string want = "(slots,) + (";
    bool same = t.dim() == 1 + (int64_t)shape.size();
    int64_t at_dim = 1, count = 1;
    for (int64_t extent : shape) {
        want += std::to_string(extent) + (at_dim < (int64_t)shape.size() ? ", " : ")");
        same = same && t.size(at_dim) == extent;
        ++at_dim;
        count *= extent;
    }
    if (!same) fail("d_state", "must have shape " + want + ", not " + shape_text(t.sizes()));
    same_kind(t, "d_state", type, like);
    int64_t step = 1;
    for (int64_t d = t.dim() - 1; d >= 1; --d) {
        if (t.size(d) > 1 && t.stride(d) != step) fail("d_state", "must have contiguous slots");
        step *= t.size(d);
    }
    *stride = t.size(0) > 1 ? t.stride(0) : count;
    if (*stride < count) fail("d_state", "must have slots of its own (no overlap)");
    *slots = held_to_int(t.size(0), "the number of slots");
}

const int* slot_of(PyObject* o, const Tensor& x, int rows_, int slots)
{
    const Tensor* t = optional(o, "slots");
    if (!t) {
        if (slots < rows_) fail("d_state", "must have a slot for each of " + std::to_string(rows_) + " rows");
        return nullptr;
    }
    if (t->dim() != 1 || t->numel() != rows_ || !t->is_contiguous()) fail("slots", "must be a contiguous 1D tensor of " + std::to_string(rows_) + " slots");
    same_kind(*t, "slots", at::kInt, x);
    return static_cast<const int*>(t->data_ptr());
}

const Tensor& step_rows(PyObject* o)
{
    const Tensor& x = main_rows(o, "d_in");
    if (x.dim() != 2) fail("d_in", "must be [rows, channels]");
    return x;
}

// conv1d_step(d_in, weight, d_state, bias, silu, slots, d_out, stream) -> d_out
PyObject* conv1d_step(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 8)) return nullptr;
    return guarded([&] {
        const Tensor& x = step_rows(v[0]);
        ssam_conv1d_step_args a{};
        filter(&a, x, v[1], v[3], v[4]);
        const Tensor& state = tensor(v[2], "d_state");
        pool(state, x.scalar_type(), x, {a.taps - 1, a.channels}, &a.slot_stride, &a.slots);
        a.d_state = state.data_ptr();
        a.rows = held_to_int(x.size(0), "the number of rows");
        a.d_slots = slot_of(v[5], x, a.rows, a.slots);
        const Tensor* given = optional(v[6], "d_out");
        const Tensor out = result(given, x, a.d_slots);
        a.in = rows(&x, "d_in", x);
        a.out = rows(&out, "d_out", x);
        call(entry.conv1d_step, a, v[7], "ssam_conv1d_step");
        if (given) {
            Py_INCREF(v[6]);
            return v[6];
        }
        return wrap(out);
    });
}

// ---- scan --------------------------------------------------------------------------------------------------------------
// in, dt, a, b, c, skip, gate, dt_bias, softplus: nine objects from v on.
template <class Args>
const Tensor& scan_inputs(Args* s, const Tensor& x, PyObject* const* v)
{
    const Tensor &a = tensor(v[2], "a"), &b = tensor(v[3], "b"), &c = tensor(v[4], "c");
    const int64_t channels = x.size(-1);
    s->dtype = code_of(x.scalar_type(), "d_in");
    if (a.dim() != 2 || a.size(0) != channels) fail("a", "must have shape (" + std::to_string(channels) + ", states), not " + shape_text(a.sizes()));
    s->d_a = dense<const float>(&a, "a", x, at::kFloat, a.sizes());
    s->b = group_rows(b, "b", x, &s->b_group);
    s->c = group_rows(c, "c", x, &s->c_group);
    if (b.sizes() != c.sizes() || b.size(-1) != a.size(1))
        fail("c", "and b must have as many groups as one another and " + std::to_string(a.size(1)) + " states");
    s->channels = held_to_int(channels, "the number of channels");
    s->states = held_to_int(a.size(1), "the number of states");
    s->groups = held_to_int(b.size(-2), "the number of groups");
    s->in = rows(&x, "d_in", x);
    s->dt = rows(&tensor(v[1], "d_dt"), "d_dt", x);
    s->d_skip = dense<const float>(optional(v[5], "skip"), "skip", x, at::kFloat, {channels});
    s->gate = rows(optional(v[6], "gate"), "gate", x);
    s->d_dt_bias = dense<const float>(optional(v[7], "dt_bias"), "dt_bias", x, at::kFloat, {channels});
    s->softplus = truth(v[8]);
    return a;
}

long long marks_of(int dtype, int channels, int states, const ssam_sequences& q)
{
    ssam_scan_selective_args s{};
    s.dtype = dtype;
    s.channels = channels;
    s.states = states;
    s.groups = 1;
    s.seq = q;
    return entry.scan_marks(&s);
}

float* marks_for(const Tensor* t, const Tensor& x, const Tensor& a, long long need)
{
    if (!t) return nullptr;
    if (t->dim() != 3 || t->size(1) != a.size(0) || t->size(2) != a.size(1) || t->size(0) < need)
        fail("d_marks", "must come from ssam_scan_selective_marks for these sequences");
    return dense<float>(t, "d_marks", x, at::kFloat, t->sizes());
}

// scan_marks(d_in, a, starts, lengths) -> d_marks
PyObject* scan_marks(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 4)) return nullptr;
    return guarded([&] {
        const Tensor &x = main_rows(v[0], "d_in"), &a = tensor(v[1], "a");
        if (a.dim() != 2 || a.size(0) != x.size(-1)) fail("a", "must have shape (" + std::to_string(x.size(-1)) + ", states), not " + shape_text(a.sizes()));
        const ssam_sequences q = sequences(x, optional(v[2], "starts"), optional(v[3], "lengths"));
        const long long count = marks_of(code_of(x.scalar_type(), "d_in"), held_to_int(a.size(0), "the number of channels"),
                                         held_to_int(a.size(1), "the number of states"), q);
        return wrap(at::empty({count, a.size(0), a.size(1)}, x.options().dtype(at::kFloat)));
    });
}

// scan(d_in, d_dt, a, b, c, skip, gate, dt_bias, softplus, d_state, d_final, d_marks, starts, lengths, d_out, d_work, stream)
//     -> d_out
PyObject* scan(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 17)) return nullptr;
    return guarded([&] {
        const Tensor& x = main_rows(v[0], "d_in");
        ssam_scan_selective_args s{};
        const Tensor& a = scan_inputs(&s, x, v);
        s.seq = sequences(x, optional(v[12], "starts"), optional(v[13], "lengths"));
        const int64_t carried[] = {s.seq.sequences, s.channels, s.states};
        s.d_state = dense<const float>(optional(v[9], "d_state"), "d_state", x, at::kFloat, carried);
        s.d_final = dense<float>(optional(v[10], "d_final"), "d_final", x, at::kFloat, carried);
        if (v[11] != Py_None) s.d_marks = marks_for(optional(v[11], "d_marks"), x, a, marks_of(s.dtype, s.channels, s.states, s.seq));
        const Tensor* given = optional(v[14], "d_out");
        const Tensor out = result(given, x, s.seq.d_begin || s.seq.d_end);
        s.out = rows(&out, "d_out", x);
        const Tensor work = workspace(entry.scan_bytes(&s), optional(v[15], "d_work"), x);
        if (work.defined()) {
            s.d_work = work.data_ptr();
            s.work_bytes = work.nbytes();
        }
        call(entry.scan, s, v[16], "ssam_scan_selective");
        if (given) {
            Py_INCREF(v[14]);
            return v[14];
        }
        return wrap(out);
    });
}

// scan_bytes(d_in, a, groups, starts, lengths) -> bytes of workspace
PyObject* scan_bytes(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 5)) return nullptr;
    return guarded([&] {
        const Tensor &x = main_rows(v[0], "d_in"), &a = tensor(v[1], "a");
        if (a.dim() != 2) fail("a", "must have shape (channels, states)");
        ssam_scan_selective_args s{};
        s.dtype = code_of(x.scalar_type(), "d_in");
        s.channels = held_to_int(a.size(0), "the number of channels");
        s.states = held_to_int(a.size(1), "the number of states");
        s.groups = (int)PyLong_AsLong(v[2]);
        if (PyErr_Occurred()) throw 0;
        s.seq = sequences(x, optional(v[3], "starts"), optional(v[4], "lengths"));
        return PyLong_FromSize_t(entry.scan_bytes(&s));
    });
}

// scan_backward(d_grad, d_in, d_dt, a, b, c, skip, gate, dt_bias, softplus, d_marks, d_grad_final, starts, lengths, state_grad, d_work,
//     stream) -> (x, dt, a, b, c, skip, gate, dt_bias, state)
PyObject* scan_backward(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 17)) return nullptr;
    return guarded([&] {
        const Tensor& x = main_rows(v[1], "d_in");
        ssam_scan_selective_backward_args s{};
        const Tensor& a = scan_inputs(&s, x, v + 1);
        s.seq = sequences(x, optional(v[12], "starts"), optional(v[13], "lengths"));
        s.grad_out = rows(&tensor(v[0], "d_grad"), "d_grad", x);
        s.d_marks = marks_for(&tensor(v[10], "d_marks"), x, a, marks_of(s.dtype, s.channels, s.states, s.seq));
        const int64_t carried[] = {s.seq.sequences, s.channels, s.states};
        s.d_grad_final = dense<const float>(optional(v[11], "d_grad_final"), "d_grad_final", x, at::kFloat, carried);
        const bool ragged = s.seq.d_begin || s.seq.d_end;
        const auto f32 = x.options().dtype(at::kFloat);
        const Tensor &b = tensor(v[4], "b"), &c = tensor(v[5], "c");
        const Tensor gx = result(nullptr, x, ragged), gdt = result(nullptr, x, ragged);
        const Tensor gb = result(nullptr, b, ragged), gc = result(nullptr, c, ragged);
        const Tensor gz = s.gate.d || v[7] != Py_None ? result(nullptr, x, ragged) : Tensor();
        const Tensor ga = at::empty(a.sizes(), f32), gk = v[6] != Py_None ? at::empty({s.channels}, f32) : Tensor();
        const Tensor gd = v[8] != Py_None ? at::empty({s.channels}, f32) : Tensor(), gs = truth(v[14]) ? at::empty(carried, f32) : Tensor();
        long long apart;
        s.grad_in = rows(&gx, "x", x);
        s.grad_dt = rows(&gdt, "dt", x);
        if (gz.defined()) s.grad_gate = rows(&gz, "gate", x);
        s.grad_b = group_rows(gb, "b", x, &apart);
        s.grad_c = group_rows(gc, "c", x, &apart);
        s.d_grad_a = static_cast<float*>(ga.data_ptr());
        if (gk.defined()) s.d_grad_skip = static_cast<float*>(gk.data_ptr());
        if (gd.defined()) s.d_grad_dt_bias = static_cast<float*>(gd.data_ptr());
        if (gs.defined()) s.d_grad_state = static_cast<float*>(gs.data_ptr());
        const Tensor work = workspace(entry.scan_backward_bytes(&s), optional(v[15], "d_work"), x);
        if (work.defined()) {
            s.d_work = work.data_ptr();
            s.work_bytes = work.nbytes();
        }
        call(entry.scan_backward, s, v[16], "ssam_scan_selective_backward");
        return Py_BuildValue("(NNNNNNNNN)", wrap(gx), wrap(gdt), wrap(ga), wrap(gb), wrap(gc), wrap(gk), wrap(gz), wrap(gd), wrap(gs));
    });
}

// scan_step(d_in, d_dt, a, b, c, skip, gate, dt_bias, softplus, d_state, slots, d_out, stream) -> d_out
PyObject* scan_step(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 13)) return nullptr;
    return guarded([&] {
        const Tensor& x = step_rows(v[0]);
        ssam_scan_selective_step_args s{};
        scan_inputs(&s, x, v);
        const Tensor& state = tensor(v[9], "d_state");
        pool(state, at::kFloat, x, {s.channels, s.states}, &s.slot_stride, &s.slots);
        s.d_state = static_cast<float*>(state.data_ptr());
        s.rows = held_to_int(x.size(0), "the number of rows");
        s.d_slots = slot_of(v[10], x, s.rows, s.slots);
        const Tensor* given = optional(v[11], "d_out");
        const Tensor out = result(given, x, s.d_slots);
        s.out = rows(&out, "d_out", x);
        call(entry.scan_step, s, v[12], "ssam_scan_selective_step");
        if (given) {
            Py_INCREF(v[11]);
            return v[11];
        }
        return wrap(out);
    });
}

// ---- scan with matrix states -------------------------------------------------------------------------------------------
const Tensor& main_heads(PyObject* o)
{
    const Tensor& t = tensor(o, "d_v");
    if (!t.is_cuda()) fail("d_v", "must live in GPU memory");
    if (t.dim() != 3 && t.dim() != 4) fail("d_v", "must be [rows, heads, width] or [sequences, rows, heads, width]");
    return t;
}

// Rows of heads: v's type, device and leading extents, a head's elements contiguous.
ssam_rows head_rows(const Tensor& t, const char* name, const Tensor& v, int64_t heads, int64_t width, long long* apart)
{
    same_kind(t, name, v.scalar_type(), v);
    const auto lead = v.sizes().slice(0, v.dim() - 2);
    if (t.dim() != v.dim() || t.sizes().slice(0, lead.size()) != lead || t.size(-2) != heads || t.size(-1) != width)
        fail(name, "must have shape " + shape_text(lead) + " + (" + std::to_string(heads) + ", " + std::to_string(width) + "), not " + shape_text(t.sizes()));
    const auto s = t.strides();
    if (s.back() != 1 && t.sizes().back() != 1) fail(name, "must have contiguous elements of a head (stride 1)");
    *apart = s[s.size() - 2];
    return s.size() == 3 ? ssam_rows{t.data_ptr(), 0, s[0]} : ssam_rows{t.data_ptr(), s[0], s[1]};
}
// A float for every row and head.
ssam_rows head_values(const Tensor* t, const char* name, const Tensor& v)
{
    if (!t) return ssam_rows{nullptr, 0, 0};
    const auto want = v.sizes().slice(0, v.dim() - 1);
    if (t->sizes() != want) fail(name, "must have shape " + shape_text(want) + ", not " + shape_text(t->sizes()));
    same_kind(*t, name, at::kFloat, v);
    const auto s = t->strides();
    if (s.back() != 1 && t->sizes().back() != 1) fail(name, "must have contiguous heads (stride 1)");
    return s.size() == 2 ? ssam_rows{t->data_ptr(), 0, s[0]} : ssam_rows{t->data_ptr(), s[0], s[1]};
}

// q, k, v, g, beta: five objects from v on; scale, unit.
template <class Args>
const Tensor& delta_inputs(Args* s, PyObject* const* o, PyObject* scale, PyObject* unit)
{
    const Tensor &k = tensor(o[1], "d_k"), &v = main_heads(o[2]);
    s->dtype = code_of(v.scalar_type(), "d_v");
    s->heads = held_to_int(v.size(-2), "the number of heads");
    s->value_dim = held_to_int(v.size(-1), "a value's width");
    if (k.dim() != v.dim()) fail("d_k", "must have as many dimensions as d_v, not shape " + shape_text(k.sizes()));
    s->key_heads = held_to_int(k.size(-2), "the number of key heads");
    s->key_dim = held_to_int(k.size(-1), "a key's width");
    s->q = head_rows(tensor(o[0], "d_q"), "d_q", v, s->key_heads, s->key_dim, &s->q_head);
    s->k = head_rows(k, "d_k", v, s->key_heads, s->key_dim, &s->k_head);
    s->v = head_rows(v, "d_v", v, s->heads, s->value_dim, &s->v_head);
    s->g = head_values(optional(o[3], "g"), "g", v);
    s->beta = head_values(&tensor(o[4], "beta"), "beta", v);
    s->unit = truth(unit);
    if (scale == Py_None) {
        s->scale = 1.0f / std::sqrt((float)(s->key_dim > 0 ? s->key_dim : 1));
    } else {
        s->scale = (float)PyFloat_AsDouble(scale);
        if (PyErr_Occurred()) throw 0;
    }
    return v;
}

long long delta_marks_of(const Tensor& k, const Tensor& v, const ssam_sequences& q)
{
    ssam_scan_delta_args s{};
    s.dtype = code_of(v.scalar_type(), "d_v");
    s.heads = held_to_int(v.size(-2), "the number of heads");
    s.key_heads = held_to_int(k.size(-2), "the number of key heads");
    s.key_dim = held_to_int(k.size(-1), "a key's width");
    s.value_dim = held_to_int(v.size(-1), "a value's width");
    s.seq = q;
    return entry.delta_marks(&s);
}

float* delta_marks_for(const Tensor* t, const Tensor& k, const Tensor& v, const ssam_sequences& q)
{
    if (!t) return nullptr;
    if (t->dim() != 4 || t->size(0) < delta_marks_of(k, v, q) || t->size(1) != v.size(-2) || t->size(2) != k.size(-1) + SSAM_DELTA_ROWS || t->size(3) != v.size(-1))
        fail("d_marks", "must come from ssam_scan_delta_marks for these sequences");
    return dense<float>(t, "d_marks", v, at::kFloat, t->sizes());
}

// delta_marks(d_k, d_v, starts, lengths) -> d_marks
PyObject* delta_marks(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (!arity(n, 4)) return nullptr;
    return guarded([&] {
        const Tensor &k = tensor(o[0], "d_k"), &v = main_heads(o[1]);
        if (k.dim() != v.dim()) fail("d_k", "must have as many dimensions as d_v, not shape " + shape_text(k.sizes()));
        const long long count = delta_marks_of(k, v, sequences(v, optional(o[2], "starts"), optional(o[3], "lengths"), 2));
        return wrap(at::empty({count, v.size(-2), k.size(-1) + SSAM_DELTA_ROWS, v.size(-1)}, v.options().dtype(at::kFloat)));
    });
}

// delta_bytes(d_k, d_v, starts, lengths) -> bytes of workspace
PyObject* delta_bytes(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (!arity(n, 4)) return nullptr;
    return guarded([&] {
        const Tensor &k = tensor(o[0], "d_k"), &v = main_heads(o[1]);
        if (k.dim() != v.dim()) fail("d_k", "must have as many dimensions as d_v, not shape " + shape_text(k.sizes()));
        ssam_scan_delta_args s{};
        s.dtype = code_of(v.scalar_type(), "d_v");
        s.heads = held_to_int(v.size(-2), "the number of heads");
        s.key_heads = held_to_int(k.size(-2), "the number of key heads");
        s.key_dim = held_to_int(k.size(-1), "a key's width");
        s.value_dim = held_to_int(v.size(-1), "a value's width");
        s.seq = sequences(v, optional(o[2], "starts"), optional(o[3], "lengths"), 2);
        return PyLong_FromSize_t(entry.delta_bytes(&s));
    });
}

// delta(d_q, d_k, d_v, g, beta, scale, unit, d_state, d_final, d_marks, starts, lengths, d_out, d_work, stream) -> d_out
PyObject* delta(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (!arity(n, 15)) return nullptr;
    return guarded([&] {
        ssam_scan_delta_args s{};
        const Tensor& v = delta_inputs(&s, o, o[5], o[6]);
        s.seq = sequences(v, optional(o[10], "starts"), optional(o[11], "lengths"), 2);
        const int64_t carried[] = {s.seq.sequences, s.heads, s.key_dim, s.value_dim};
        s.d_state = dense<const float>(optional(o[7], "d_state"), "d_state", v, at::kFloat, carried);
        s.d_final = dense<float>(optional(o[8], "d_final"), "d_final", v, at::kFloat, carried);
        s.d_marks = delta_marks_for(optional(o[9], "d_marks"), tensor(o[1], "d_k"), v, s.seq);
        const Tensor* given = optional(o[12], "d_out");
        const Tensor out = result(given, v, s.seq.d_begin || s.seq.d_end);
        s.out = head_rows(out, "d_out", v, s.heads, s.value_dim, &s.out_head);
        const Tensor work = workspace(entry.delta_bytes(&s), optional(o[13], "d_work"), v);
        if (work.defined()) {
            s.d_work = work.data_ptr();
            s.work_bytes = work.nbytes();
        }
        call(entry.delta, s, o[14], "ssam_scan_delta");
        if (given) {
            Py_INCREF(o[12]);
            return o[12];
        }
        return wrap(out);
    });
}

// delta_backward(d_grad, d_q, d_k, d_v, g, beta, scale, unit, d_marks, d_grad_final, starts, lengths, state_grad, d_work, stream)
//     -> (q, k, v, g, beta, state)
PyObject* delta_backward(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (!arity(n, 15)) return nullptr;
    return guarded([&] {
        ssam_scan_delta_backward_args s{};
        const Tensor& v = delta_inputs(&s, o + 1, o[6], o[7]);
        s.seq = sequences(v, optional(o[10], "starts"), optional(o[11], "lengths"), 2);
        s.grad_out = head_rows(tensor(o[0], "d_grad"), "d_grad", v, s.heads, s.value_dim, &s.grad_out_head);
        const Tensor &q = tensor(o[1], "d_q"), &k = tensor(o[2], "d_k"), &beta = tensor(o[5], "beta");
        s.d_marks = delta_marks_for(&tensor(o[8], "d_marks"), k, v, s.seq);
        const int64_t carried[] = {s.seq.sequences, s.heads, s.key_dim, s.value_dim};
        s.d_grad_final = dense<const float>(optional(o[9], "d_grad_final"), "d_grad_final", v, at::kFloat, carried);
        const bool ragged = s.seq.d_begin || s.seq.d_end;
        const Tensor gq = result(nullptr, q, ragged), gk = result(nullptr, k, ragged), gv = result(nullptr, v, ragged), gb = result(nullptr, beta, ragged);
        const Tensor gg = o[4] != Py_None ? result(nullptr, beta, ragged) : Tensor();
        const Tensor gs = truth(o[12]) ? at::empty(carried, beta.options()) : Tensor();
        long long apart;
        s.grad_q = head_rows(gq, "q", v, s.key_heads, s.key_dim, &apart);
        s.grad_k = head_rows(gk, "k", v, s.key_heads, s.key_dim, &apart);
        s.grad_v = head_rows(gv, "v", v, s.heads, s.value_dim, &apart);
        if (gg.defined()) s.grad_g = head_values(&gg, "g", v);
        s.grad_beta = head_values(&gb, "beta", v);
        if (gs.defined()) s.d_grad_state = static_cast<float*>(gs.data_ptr());
        const Tensor work = workspace(entry.delta_backward_bytes(&s), optional(o[13], "d_work"), v);
        if (work.defined()) {
            s.d_work = work.data_ptr();
            s.work_bytes = work.nbytes();
        }
        call(entry.delta_backward, s, o[14], "ssam_scan_delta_backward");
        return Py_BuildValue("(NNNNNN)", wrap(gq), wrap(gk), wrap(gv), wrap(gg), wrap(gb), wrap(gs));
    });
}

// delta_step(d_q, d_k, d_v, g, beta, d_state, scale, unit, slots, d_out, stream) -> d_out
PyObject* delta_step(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (!arity(n, 11)) return nullptr;
    return guarded([&] {
        ssam_scan_delta_step_args s{};
        const Tensor& v = delta_inputs(&s, o, o[6], o[7]);
        if (v.dim() != 3) fail("d_v", "must be [rows, heads, width]");
        const Tensor& state = tensor(o[5], "d_state");
        pool(state, at::kFloat, v, {s.heads, s.key_dim, s.value_dim}, &s.slot_stride, &s.slots);
        s.d_state = static_cast<float*>(state.data_ptr());
        s.rows = held_to_int(v.size(0), "the number of rows");
        s.d_slots = slot_of(o[8], v, s.rows, s.slots);
        const Tensor* given = optional(o[9], "d_out");
        const Tensor out = result(given, v, s.d_slots);
        s.out = head_rows(out, "d_out", v, s.heads, s.value_dim, &s.out_head);
        call(entry.delta_step, s, o[10], "ssam_scan_delta_step");
        if (given) {
            Py_INCREF(o[9]);
            return o[9];
        }
        return wrap(out);
    });
}

// ---- norm ----------------------------------------------------------------------------------------------------------------
// d_in; weight, groups, eps.
template <class Args>
const Tensor& norm_inputs(Args* a, PyObject* in, PyObject* weight, PyObject* groups, PyObject* eps)
{
    const Tensor& x = main_rows(in, "d_in");
    a->dtype = a->param_dtype = code_of(x.scalar_type(), "d_in");
    a->channels = held_to_int(x.size(-1), "the number of channels");
    const long many = PyLong_AsLong(groups);
    if (PyErr_Occurred()) throw 0;
    if (many < 1 || many > a->channels || a->channels % many) fail("groups", "must divide the " + std::to_string(a->channels) + " channels");
    a->groups = (int)many;
    a->eps = (float)PyFloat_AsDouble(eps);
    if (PyErr_Occurred()) throw 0;
    a->sequences = x.dim() == 3 ? held_to_int(x.size(0), "the number of sequences") : 1;
    a->rows = held_to_int(x.size(-2), "the number of rows");
    a->in = rows(&x, "d_in", x);
    if (const Tensor* w = optional(weight, "weight")) {
        if (w->scalar_type() != x.scalar_type() && w->scalar_type() != at::kFloat) fail("weight", "must be " + type_text(x.scalar_type()) + " or torch.float32");
        a->param_dtype = code_of(w->scalar_type(), "weight");
        a->d_weight = dense(w, "weight", x, w->scalar_type(), {a->channels / a->groups});
    }
    return x;
}

// d_residual, d_sum, gate: three objects from v on.
const Tensor& norm_all(ssam_rms_norm_args* a, PyObject* in, PyObject* weight, PyObject* const* v, PyObject* groups, PyObject* eps)
{
    const Tensor& x = norm_inputs(a, in, weight, groups, eps);
    a->residual = rows(optional(v[0], "d_residual"), "d_residual", x);
    if (v[1] != Py_None && v[0] == Py_None) fail("d_sum", "belongs to a d_residual");
    a->sum = rows(optional(v[1], "d_sum"), "d_sum", x);
    a->gate = rows(optional(v[2], "gate"), "gate", x);
    return x;
}

// norm(d_in, weight, d_residual, d_sum, gate, groups, eps, d_out, stream) -> d_out
PyObject* norm(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 9)) return nullptr;
    return guarded([&] {
        ssam_rms_norm_args a{};
        const Tensor& x = norm_all(&a, v[0], v[1], v + 2, v[5], v[6]);
        const Tensor* given = optional(v[7], "d_out");
        const Tensor out = result(given, x, false);
        a.out = rows(&out, "d_out", x);
        call(entry.norm, a, v[8], "ssam_rms_norm");
        if (given) {
            Py_INCREF(v[7]);
            return v[7];
        }
        return wrap(out);
    });
}

// norm_e4m3(d_in, weight, d_residual, d_sum, gate, groups, eps, block, d_out, d_scales, stream) -> (values, scales)
PyObject* norm_e4m3(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 11)) return nullptr;
    return guarded([&] {
        ssam_rms_norm_args a{};
        const Tensor& x = norm_all(&a, v[0], v[1], v + 2, v[5], v[6]);
        const int width = a.channels / a.groups;
        a.block = width;
        if (v[7] != Py_None) {
            const long block = PyLong_AsLong(v[7]);
            if (PyErr_Occurred()) throw 0;
            if (block < 1 || block > width || width % block || (block < 16 && block != width))
                fail("block", "must divide the " + std::to_string(width) + " channels of a group, and be 16 at least or all of them");
            a.block = (int)block;
        }
        const Tensor *given = optional(v[8], "d_out"), *given_scales = optional(v[9], "d_scales");
        const Tensor out = given ? *given : at::empty(x.sizes(), x.options().dtype(at::kFloat8_e4m3fn));
        if (out.sizes() != x.sizes()) fail("d_out", "must have shape " + shape_text(x.sizes()) + ", not " + shape_text(out.sizes()));
        same_kind(out, "d_out", at::kFloat8_e4m3fn, x);
        const auto s = out.strides();
        if (s.back() != 1 && out.sizes().back() != 1) fail("d_out", "must have contiguous channels (stride 1)");
        a.out = s.size() == 2 ? ssam_rows{out.data_ptr(), 0, s[0]} : ssam_rows{out.data_ptr(), s[0], s[1]};
        std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = a.channels / a.block;
        const Tensor scales = given_scales ? *given_scales : at::empty(shape, x.options().dtype(at::kFloat));
        a.d_scales = dense<float>(&scales, "d_scales", x, at::kFloat, shape);
        call(entry.norm_e4m3, a, v[10], "ssam_rms_norm_e4m3");
        return Py_BuildValue("(NN)", wrap(out), wrap(scales));
    });
}

// norm_backward(d_grad, d_in, weight, d_grad_sum, gate, groups, eps, d_work, stream) -> (x, weight, gate)
PyObject* norm_backward(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 9)) return nullptr;
    return guarded([&] {
        ssam_rms_norm_backward_args a{};
        const Tensor& x = norm_inputs(&a, v[1], v[2], v[5], v[6]);
        a.grad_out = rows(&tensor(v[0], "d_grad"), "d_grad", x);
        a.grad_sum = rows(optional(v[3], "d_grad_sum"), "d_grad_sum", x);
        a.gate = rows(optional(v[4], "gate"), "gate", x);
        const Tensor gx = result(nullptr, x, false), gz = v[4] != Py_None ? result(nullptr, x, false) : Tensor();
        const Tensor gw = v[2] != Py_None ? at::empty({a.channels / a.groups}, tensor(v[2], "weight").options()) : Tensor();
        a.grad_in = rows(&gx, "x", x);
        if (gz.defined()) a.grad_gate = rows(&gz, "gate", x);
        if (gw.defined()) a.d_grad_weight = gw.data_ptr();
        const Tensor work = workspace(entry.norm_backward_bytes(&a), optional(v[7], "d_work"), x);
        if (work.defined()) {
            a.d_work = work.data_ptr();
            a.work_bytes = work.nbytes();
        }
        call(entry.norm_backward, a, v[8], "ssam_rms_norm_backward");
        return Py_BuildValue("(NNN)", wrap(gx), wrap(gw), wrap(gz));
    });
}

// bind(exception class, addresses of the entry points in the order of `entry`)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    constexpr int kCount = sizeof(entry) / sizeof(void*);
    static_assert(sizeof(void*) == sizeof(entry.conv1d));
    if (!arity(n, 1 + kCount)) return nullptr;
    void* p[kCount];
    for (int i = 0; i < kCount; ++i) p[i] = PyLong_AsVoidPtr(v[i + 1]);
    if (PyErr_Occurred()) return nullptr;
    Py_INCREF(v[0]);
    Py_XDECREF(status_error);
    status_error = v[0];
    std::memcpy(&entry, p, sizeof(entry));       // nothing but pointers
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind), FAST(conv1d), FAST(conv1d_backward), FAST(conv1d_step), FAST(scan), FAST(scan_bytes), FAST(scan_marks),
                         FAST(scan_backward), FAST(scan_step), FAST(delta), FAST(delta_bytes), FAST(delta_marks), FAST(delta_step), FAST(norm),
                         FAST(norm_e4m3), FAST(norm_backward), FAST(delta_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sequence", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sequence(void) { return PyModule_Create(&module); }
