// Argument marshalling of the Python binding for the sequence operators: shapes, types, devices and strides of the tensors are
// checked and put into the C ABI's structs here.  In Python the dozen tensors of a call cost 9 us, more than its kernel; here one
// is looked at through its C++ object, and the call costs 1 to 2 us besides the launch.  Computes nothing.  The interpreter lock is
// released around the call, as in ssam_marshal.c.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/Functions.h>

#include <stdexcept>
#include <string>

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
    return t == at::kFloat ? "torch.float32" : t == at::kHalf ? "torch.float16" : t == at::kBFloat16 ? "torch.bfloat16" : t == at::kInt ? "torch.int32" : c10::toString(t);
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

ssam_sequences sequences(const Tensor& like, const Tensor* starts, const Tensor* lengths)
{
    if (starts && lengths) fail("starts", "and lengths exclude one another");
    ssam_sequences q{1, held_to_int(like.size(-2), "the number of rows"), nullptr, nullptr};
    if (like.dim() == 2) {
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

// bind(exception class, addresses of the ten entry points in the order of `entry`)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (!arity(n, 11)) return nullptr;
    void* p[10];
    for (int i = 0; i < 10; ++i) p[i] = PyLong_AsVoidPtr(v[i + 1]);
    if (PyErr_Occurred()) return nullptr;
    Py_INCREF(v[0]);
    Py_XDECREF(status_error);
    status_error = v[0];
    entry.conv1d = (decltype(entry.conv1d))p[0];
    entry.conv1d_backward = (decltype(entry.conv1d_backward))p[1];
    entry.conv1d_backward_bytes = (decltype(entry.conv1d_backward_bytes))p[2];
    entry.conv1d_step = (decltype(entry.conv1d_step))p[3];
    entry.scan = (decltype(entry.scan))p[4];
    entry.scan_bytes = (decltype(entry.scan_bytes))p[5];
    entry.scan_marks = (decltype(entry.scan_marks))p[6];
    entry.scan_backward = (decltype(entry.scan_backward))p[7];
    entry.scan_backward_bytes = (decltype(entry.scan_backward_bytes))p[8];
    entry.scan_step = (decltype(entry.scan_step))p[9];
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind), FAST(conv1d), FAST(conv1d_backward), FAST(conv1d_step), FAST(scan), FAST(scan_bytes), FAST(scan_marks),
                         FAST(scan_backward), FAST(scan_step), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sequence", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sequence(void) { return PyModule_Create(&module); }
