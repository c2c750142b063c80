// The sequence operators on torch tensors: a Python module that checks the tensors, allocates results and calls the C ABI of libxl_seq.
//
// A call of one token keeps the GPU busy for 2 to 6 us.  Looking at a dozen tensors from Python takes longer than that; here it takes a microsecond,
// and what is left of a call is its allocations and the launch.
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/hip/HIPStream.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <sstream>
#include <string>
#include <type_traits>

#include "seq_overlap.h"
#include "xl_seq.h"

namespace {

// Addresses of the library's functions and the exception that a refusal raises: set once by bind().
decltype(&xl_causal_conv) g_conv;
decltype(&xl_selective_scan) g_scan;
decltype(&xl_selective_scan_workspace) g_scan_workspace;
decltype(&xl_quantize_blocks) g_quantize;
decltype(&xl_block_matmul) g_matmul;
decltype(&xl_rms_norm) g_norm;
decltype(&xl_add_adapters) g_adapters;
decltype(&xl_add_adapters_workspace) g_adapters_workspace;
decltype(&xl_gated_delta_rule) g_delta;
decltype(&xl_gated_delta_rule_workspace) g_delta_workspace;
decltype(&xl_seq_last_error) g_last_error;
PyObject *g_error;

struct Refused {
    xl_status status;
    std::string message;
};

template <typename... Args> [[noreturn]] void refuse(xl_status status, const Args &...args)
{
    std::ostringstream s;
    (s << ... << args);
    throw Refused{status, s.str()};
}

// Where tensors lie: rows of [batch, length, width], a contiguous block (or nothing), rows of [rows, k] that take `width` bytes each, and single numbers of [rows, columns].
int64_t address(const at::Tensor &t) { return reinterpret_cast<int64_t>(t.data_ptr()); }
xls::Span rows_of(const at::Tensor &t)
{
    const int64_t size = t.element_size();
    return {address(t), t.size(0), t.size(1), t.stride(0) * size, t.stride(1) * size, t.size(2) * size};
}
// rows of [batch, length, heads, width]; heads that lie apart as if what lies between them were theirs
xls::Span heads_of(const at::Tensor &t)
{
    const int64_t size = t.element_size();
    return {address(t), t.size(0), t.size(1), t.stride(0) * size, t.stride(1) * size, t.size(2) > 0 ? ((t.size(2) - 1) * t.stride(2) + t.size(3)) * size : 0};
}
xls::Span block_of(const at::Tensor *t) { return t ? xls::Span{address(*t), 1, 1, 0, 0, int64_t(t->nbytes())} : xls::Span{}; }
xls::Span rows_of(const at::Tensor &t, int64_t width) { return {address(t), 1, t.size(0), 0, t.stride(0) * int64_t(t.element_size()), width}; }
xls::Span numbers_of(const at::Tensor &t)
{
    const int64_t size = t.element_size();
    return {address(t), t.size(0), t.size(1), t.stride(0) * size, t.stride(1) * size, size};
}
struct Named {
    const char *what;
    xls::Span span;
};

// One call: on the device of its first tensor, which is the current one for as long.
struct Op {
    const char *name;
    const at::Tensor &first;
    const c10::DeviceGuard guard;
    const c10::DeviceIndex device;

    Op(const char *name, const at::Tensor &first) : name(name), first(first), guard(on_gpu(name, first)), device(first.get_device()) {}

    static c10::Device on_gpu(const char *name, const at::Tensor &t)
    {
        if (!t.is_cuda()) refuse(XL_E_DEVICE, name, ": tensors must be on a GPU (there is no CPU path)");
        return t.device();
    }

    // A result: from the allocator that an empty tensor's memory comes from (not from that of the inputs, which may be of other kinds of memory), without the way through the
    // dispatcher (0.4 us).
    c10::Allocator *allocator() const
    {
        static c10::Allocator *const own = [this] {
            const c10::impl::ExcludeDispatchKeyGuard no_modes(c10::python_ks);      // that would make a tensor of another kind
            return at::empty({0}, first.options().dtype(at::kByte)).storage().allocator();
        }();
        return own;
    }
    at::Tensor make(at::IntArrayRef shape, at::ScalarType type) const
    {
        return at::Tensor(at::detail::empty_generic(shape, allocator(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt));
    }
    at::Tensor make(at::IntArrayRef shape, at::IntArrayRef steps, at::ScalarType type) const
    {
        return at::Tensor(at::detail::empty_strided_generic(shape, steps, allocator(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type));
    }

    // On the device, of the type and shape, no gradient asked for, backwards or forwards.
    void check(const char *what, const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape) const
    {
        if (!t.is_cuda() || t.get_device() != device) refuse(XL_E_DEVICE, name, ": ", what, " is on ", t.device(), ", not on cuda:", int(device));
        if (t.scalar_type() != type) refuse(XL_E_UNSUPPORTED, name, ": ", what, " is ", t.scalar_type(), ", not ", type);
        if (t.sizes() != shape) refuse(XL_E_SHAPE, name, ": ", what, " has shape ", t.sizes(), ", not ", shape);
        if (t.is_neg()) refuse(XL_E_UNSUPPORTED, name, ": ", what, " is a view of numbers that are to be negated (resolve_neg makes a tensor of it)");
        if (t.requires_grad() && c10::GradMode::is_enabled()) refuse(XL_E_UNSUPPORTED, name, ": ", what, " asks for a gradient: inference only");
        if (t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode()) refuse(XL_E_UNSUPPORTED, name, ": ", what, " carries a tangent: inference only");
    }

    // [batch, length, width] with a contiguous last dimension: its steps between sequences and tokens.
    void rows(const char *what, const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape, int64_t &batch, int64_t &token) const
    {
        check(what, t, type, shape);
        if (t.stride(2) != 1 && shape[2] > 1) refuse(XL_E_SHAPE, name, ": the last dimension of ", what, " must be contiguous");
        batch = t.stride(0);
        token = t.stride(1);
    }

    // [batch, length, heads, width] with a contiguous last dimension: its steps between sequences, tokens and heads.
    void heads(const char *what, const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape, long long &batch, long long &token, long long &head) const
    {
        check(what, t, type, shape);
        if (t.stride(3) != 1 && shape[3] > 1) refuse(XL_E_SHAPE, name, ": the last dimension of ", what, " must be contiguous");
        batch = t.stride(0);
        token = t.stride(1);
        head = t.stride(2);
    }

    // A contiguous tensor, or none.
    void *dense(const char *what, const at::Tensor *t, at::ScalarType type, at::IntArrayRef shape) const
    {
        if (!t) return nullptr;
        check(what, *t, type, shape);
        if (!t->is_contiguous()) refuse(XL_E_SHAPE, name, ": ", what, " must be contiguous");
        return t->data_ptr();
    }
    template <typename T> T *dense_as(const char *what, const at::Tensor *t, at::ScalarType type, at::IntArrayRef shape) const
    {
        return static_cast<T *>(dense(what, t, type, shape));
    }

    // A tensor of the caller's that the call writes: every number in a place of its own, apart from what the call reads and writes otherwise.
    void apart(const char *what, const xls::Span &written, std::initializer_list<Named> others) const
    {
        if (xls::overlaps_itself(written)) refuse(XL_E_SHAPE, name, ": rows of ", what, " share memory with each other");
        for (const Named &o : others)
            if (xls::overlap(written, o.span)) refuse(XL_E_SHAPE, name, ": ", what, " shares memory with ", o.what);
    }

    // Enqueued on the current stream of the tensors' device.
    template <typename A> void run(xl_status (*f)(const A *, void *), const A &args) const
    {
        const xl_status st = f(&args, c10::hip::getCurrentHIPStream(device).stream());
        if (st != XL_OK) throw Refused{st, g_last_error()};
    }
};

// A tensor of the caller's has new contents: whoever has saved it for a backward pass has to find out.
void written(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

int64_t type_code(const char *name, const char *what, at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return XL_F32;
    case at::kHalf: return XL_F16;
    case at::kBFloat16: return XL_BF16;
    default: refuse(XL_E_UNSUPPORTED, name, ": ", what, " is ", t);
    }
}

// Arguments come by position from this module's only caller, the Python functions of the same names.
struct Args {
    PyObject *const *args;
    const at::Tensor &tensor(int i) const
    {
        if (!THPVariable_Check(args[i])) {
            PyErr_Format(PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(args[i])->tp_name);
            throw python_error();
        }
        return THPVariable_Unpack(args[i]);
    }
    const at::Tensor *optional(int i) const { return args[i] == Py_None ? nullptr : &tensor(i); }
    double number(int i) const
    {
        const double v = PyFloat_AsDouble(args[i]);
        if (v == -1. && PyErr_Occurred()) throw python_error();
        return v;
    }
    bool flag(int i) const
    {
        const int v = PyObject_IsTrue(args[i]);
        if (v < 0) throw python_error();
        return v;
    }
};

// A result as it goes back: the object that was handed in, or a new one.
PyObject *result(PyObject *given, const at::Tensor &t) { return given == Py_None ? THPVariable_Wrap(t) : Py_NewRef(given); }

// (first, second) as a tuple; what was handed in goes back as the object it was.
PyObject *pair(PyObject *given0, const at::Tensor &t0, PyObject *given1, const at::Tensor &t1)
{
    PyObject *a = given0 == Py_None ? THPVariable_Wrap(t0) : Py_NewRef(given0), *b = given1 == Py_None ? THPVariable_Wrap(t1) : Py_NewRef(given1);
    PyObject *both = a && b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    if (!both) throw python_error();
    return both;
}

PyObject *raised(const Refused &r)
{
    PyObject *e = PyObject_CallFunction(g_error, "is", int(r.status), r.message.c_str());
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

// The state that a call leaves: the one handed in, the cache itself, or a new one.
const at::Tensor *state_out(const Op &op, const at::Tensor *state, const at::Tensor *new_state, const at::Tensor *slots)
{
    if (slots && !state) refuse(XL_E_SHAPE, op.name, ": slots name rows of a state, and none is given");
    return new_state ? new_state : slots ? state : nullptr;
}

PyObject *causal_conv(const Args &in)       // x, weight, bias, silu, state, new_state, lengths, slots, out
{
    const at::Tensor &x = in.tensor(0), &weight = in.tensor(1);
    const at::Tensor *bias = in.optional(2), *state = in.optional(4), *lengths = in.optional(6), *slots = in.optional(7), *given = in.optional(8);
    if (x.dim() != 3 || weight.dim() != 2) refuse(XL_E_SHAPE, "causal_conv: x is [batch, length, channels] and weight [channels, taps]");
    const Op op("causal_conv", x);
    const at::ScalarType type = x.scalar_type();
    xl_causal_conv_args a = {};
    a.dtype = type_code(op.name, "x", type);
    a.batch = x.size(0);
    a.length = x.size(1);
    a.channels = x.size(2);
    a.taps = weight.size(1);
    a.silu = in.flag(3);
    const at::Tensor *kept = state_out(op, state, in.optional(5), slots);
    a.nslots = slots && state->dim() ? state->size(0) : a.batch;
    const int64_t shape[] = {a.nslots, a.taps > 0 ? a.taps - 1 : 0, a.channels};
    at::Tensor made, made_state;
    if (!given) given = &(made = op.make(x.sizes(), type));
    if (!kept) kept = &(made_state = op.make(shape, type));
    int64_t b, t;
    op.rows("x", x, type, x.sizes(), b, t);
    a.x_batch = b, a.x_token = t;
    op.rows("out", *given, type, x.sizes(), b, t);
    a.y_batch = b, a.y_token = t;
    a.x = x.data_ptr();
    a.weight = op.dense_as<float>("weight", &weight, at::kFloat, {a.channels, a.taps});
    a.bias = op.dense_as<float>("bias", bias, at::kFloat, {a.channels});
    a.state = op.dense("state", state, type, shape);
    a.new_state = op.dense("new_state", kept, type, shape);
    a.lengths = op.dense_as<int>("lengths", lengths, at::kInt, {a.batch});
    a.slots = op.dense_as<int>("slots", slots, at::kInt, {a.batch});
    a.y = given->data_ptr();
    if (given != &made || kept != &made_state) {
        const Named old = {"state (or is it, as a whole)", a.state != a.new_state ? block_of(state) : xls::Span{}}, input = {"x", rows_of(x)};
        const Named shared[] = {{"weight", block_of(&weight)}, {"bias", block_of(bias)}, {"lengths", block_of(lengths)}, {"slots", block_of(slots)}};
        if (given != &made) op.apart("out", rows_of(*given), {input, old, {"new_state", block_of(kept)}, shared[0], shared[1], shared[2], shared[3]});
        if (kept != &made_state) op.apart("new_state", block_of(kept), {input, old, shared[0], shared[1], shared[2], shared[3]});
    }
    op.run(g_conv, a);
    if (given != &made) written(*given);
    if (kept != &made_state) written(*kept);
    return pair(in.args[8], *given, in.args[5] == Py_None && slots ? in.args[4] : in.args[5], *kept);
}

PyObject *selective_scan(const Args &in)    // u, delta, A, B, C, D, z, delta_bias, softplus, state, new_state, lengths, slots, out
{
    const at::Tensor &u = in.tensor(0), &delta = in.tensor(1), &A = in.tensor(2), &B = in.tensor(3), &C = in.tensor(4);
    const at::Tensor *D = in.optional(5), *z = in.optional(6), *delta_bias = in.optional(7), *state = in.optional(9), *lengths = in.optional(11),
                     *slots = in.optional(12), *given = in.optional(13);
    if (u.dim() != 3 || A.dim() != 2) refuse(XL_E_SHAPE, "selective_scan: u is [batch, length, channels] and A [channels, states]");
    const Op op("selective_scan", u);
    const at::ScalarType type = u.scalar_type();
    xl_scan_args a = {};
    a.dtype = type_code(op.name, "u", type);
    a.batch = u.size(0);
    a.length = u.size(1);
    a.channels = u.size(2);
    a.states = A.size(1);
    a.softplus = in.flag(8);
    const at::Tensor *kept = state_out(op, state, in.optional(10), slots);
    a.nslots = slots && state->dim() ? state->size(0) : a.batch;
    const int64_t shape[] = {a.nslots, a.channels, a.states}, wide[] = {a.batch, a.length, a.states};
    at::Tensor made, made_state;
    if (!given) given = &(made = op.make(u.sizes(), type));
    if (!kept) kept = &(made_state = op.make(shape, at::kFloat));
    int64_t b, t;
    op.rows("u", u, type, u.sizes(), b, t);
    a.u_batch = b, a.u_token = t;
    op.rows("delta", delta, type, u.sizes(), b, t);
    a.delta_batch = b, a.delta_token = t;
    if (z) {
        op.rows("z", *z, type, u.sizes(), b, t);
        a.z_batch = b, a.z_token = t;
        a.z = z->data_ptr();
    }
    op.rows("out", *given, type, u.sizes(), b, t);
    a.y_batch = b, a.y_token = t;
    op.rows("B", B, type, wide, b, t);
    a.b_batch = b, a.b_token = t;
    op.rows("C", C, type, wide, b, t);
    a.c_batch = b, a.c_token = t;
    a.u = u.data_ptr();
    a.delta = delta.data_ptr();
    a.A = op.dense_as<float>("A", &A, at::kFloat, {a.channels, a.states});
    a.B = B.data_ptr();
    a.C = C.data_ptr();
    a.D = op.dense_as<float>("D", D, at::kFloat, {a.channels});
    a.delta_bias = op.dense_as<float>("delta_bias", delta_bias, at::kFloat, {a.channels});
    a.state = op.dense_as<float>("state", state, at::kFloat, shape);
    a.new_state = op.dense_as<float>("new_state", kept, at::kFloat, shape);
    a.lengths = op.dense_as<int>("lengths", lengths, at::kInt, {a.batch});
    a.slots = op.dense_as<int>("slots", slots, at::kInt, {a.batch});
    a.y = given->data_ptr();
    if (given != &made || kept != &made_state) {
        const Named old = {"state (or is it, as a whole)", a.state != a.new_state ? block_of(state) : xls::Span{}};
        const Named shared[] = {{"A", block_of(&A)}, {"D", block_of(D)}, {"delta_bias", block_of(delta_bias)}, {"B", rows_of(B)}, {"C", rows_of(C)}, {"lengths", block_of(lengths)}, {"slots", block_of(slots)}};
        Named tokens[] = {{"u (or is it, as a whole)", rows_of(u)}, {"delta (or is it, as a whole)", rows_of(delta)}, {"z (or is it, as a whole)", z ? rows_of(*z) : xls::Span{}}};
        if (kept != &made_state)
            op.apart("new_state", block_of(kept), {tokens[0], tokens[1], tokens[2], old, shared[0], shared[1], shared[2], shared[3], shared[4], shared[5], shared[6]});
        if (given != &made) {       // may take the place of an input of its shape, as a whole: a token's numbers are read before its result is written
            const xls::Span y = rows_of(*given);
            for (Named &t : tokens)
                if (t.span == y) t.span = {};
            op.apart("out", y, {tokens[0], tokens[1], tokens[2], old, {"new_state", block_of(kept)}, shared[0], shared[1], shared[2], shared[3], shared[4], shared[5], shared[6]});
        }
    }
    at::Tensor workspace;
    a.workspace_bytes = g_scan_workspace(&a);
    if (a.workspace_bytes > 0) a.workspace = (workspace = op.make({a.workspace_bytes}, at::kByte)).data_ptr();
    op.run(g_scan, a);
    if (given != &made) written(*given);
    if (kept != &made_state) written(*kept);
    return pair(in.args[13], *given, in.args[10] == Py_None && slots ? in.args[9] : in.args[10], *kept);
}

// The memory of the last row of 8-bit numbers goes on to the next multiple of 16 bytes.
void check_readable(const Op &op, const char *what, const at::Tensor &t)
{
    const int64_t rows = t.size(0), k = t.size(1);
    if (k % 16 && rows && t.storage_offset() + (rows - 1) * t.stride(0) + (k + 15) / 16 * 16 > int64_t(t.storage().nbytes()))
        refuse(XL_E_SHAPE, op.name, ": the last row of ", what, " must have memory up to the next multiple of 16 bytes");
}

PyObject *quantize(const Args &in)          // name, x, block_rows, out, scales
{
    const char *name = PyUnicode_AsUTF8(in.args[0]);
    if (!name) throw python_error();
    const at::Tensor &x = in.tensor(1);
    const at::Tensor *out = in.optional(3), *scales = in.optional(4);
    if (x.dim() != 2) refuse(XL_E_SHAPE, name, ": x is [rows, k]");
    const Op op(name, x);
    const at::ScalarType type = x.scalar_type();
    xl_quantize_args a = {};
    a.dtype = type_code(name, "x", type);
    a.rows = x.size(0);
    a.k = x.size(1);
    a.block_rows = PyLong_AsLongLong(in.args[2]);
    if (PyErr_Occurred()) throw python_error();
    const int64_t shape[] = {(a.rows + a.block_rows - 1) / a.block_rows, (a.k + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK};
    at::Tensor made, made_scales;
    if (!out) {
        const int64_t wide = (a.k + 15) / 16 * 16;
        made = op.make({a.rows, wide}, at::kFloat8_e4m3fn);
        if (wide != a.k) made.unsafeGetTensorImpl()->set_sizes_and_strides(x.sizes(), at::IntArrayRef{wide, 1});
        out = &made;
    }
    if (!scales) {      // a column for each block: the product reads the scales of neighbouring rows together
        const int64_t step[] = {a.block_rows == 1 ? 1 : shape[1], a.block_rows == 1 ? shape[0] : 1};
        scales = &(made_scales = op.make(shape, step, at::kFloat));
    }
    op.check("x", x, type, x.sizes());
    op.check("out", *out, at::kFloat8_e4m3fn, x.sizes());
    op.check("scales", *scales, at::kFloat, shape);
    if (a.k > 1 && (x.stride(1) != 1 || out->stride(1) != 1)) refuse(XL_E_SHAPE, name, ": rows of x and out must be contiguous");
    check_readable(op, "out", *out);
    a.x_row = x.stride(0);
    a.q_row = out->stride(0);
    a.scale_row = scales->stride(0);
    a.scale_block = scales->stride(1);
    a.x = x.data_ptr();
    a.q = out->data_ptr();
    a.scales = static_cast<float *>(scales->data_ptr());
    const xls::Span input = rows_of(x, a.k * int64_t(x.element_size()));
    if (out != &made) op.apart("out", rows_of(*out, (a.k + 15) / 16 * 16), {{"x", input}, {"scales", numbers_of(*scales)}});
    if (scales != &made_scales) op.apart("scales", numbers_of(*scales), {{"x", input}});
    op.run(g_quantize, a);
    if (out != &made) written(*out);
    if (scales != &made_scales) written(*scales);
    return pair(in.args[3], *out, in.args[4], *scales);
}

PyObject *block_matmul(const Args &in)      // a, a_scales, b, b_scales, bias, dtype, out
{
    const at::Tensor &a = in.tensor(0), &a_scales = in.tensor(1), &b = in.tensor(2), &b_scales = in.tensor(3);
    const at::Tensor *bias = in.optional(4), *out = in.optional(6);
    if (a.dim() != 2 || b.dim() != 2) refuse(XL_E_SHAPE, "block_matmul: a is [m, k] and b [n, k]");
    const Op op("block_matmul", a);
    if (!out && !THPDtype_Check(in.args[5])) {
        PyErr_SetString(PyExc_TypeError, "block_matmul: dtype must be a torch.dtype");
        throw python_error();
    }
    const at::ScalarType type = out ? out->scalar_type() : reinterpret_cast<THPDtype *>(in.args[5])->scalar_type;
    xl_block_matmul_args g = {};
    g.dtype = type_code(op.name, "the result", type);
    g.m = a.size(0);
    g.k = a.size(1);
    g.n = b.size(0);
    const int64_t shape[] = {g.m, g.n}, blocks = (g.k + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK;
    at::Tensor made;
    if (out) op.check("out", *out, type, shape);
    else out = &(made = op.make(shape, type));
    op.check("a", a, at::kFloat8_e4m3fn, a.sizes());
    op.check("b", b, at::kFloat8_e4m3fn, {g.n, g.k});
    op.check("a_scales", a_scales, at::kFloat, {g.m, blocks});
    op.check("b_scales", b_scales, at::kFloat, {(g.n + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK, blocks});
    if ((g.k > 1 && (a.stride(1) != 1 || b.stride(1) != 1)) || (g.n > 1 && out->stride(1) != 1))
        refuse(XL_E_SHAPE, "block_matmul: rows of a, b and out must be contiguous");
    check_readable(op, "a", a);
    check_readable(op, "b", b);
    g.a_row = a.stride(0);
    g.b_row = b.stride(0);
    g.a_scale_row = a_scales.stride(0);
    g.a_scale_block = a_scales.stride(1);
    g.b_scale_row = b_scales.stride(0);
    g.b_scale_block = b_scales.stride(1);
    g.y_row = out->stride(0);
    g.a = a.data_ptr();
    g.b = b.data_ptr();
    g.a_scales = static_cast<const float *>(a_scales.data_ptr());
    g.b_scales = static_cast<const float *>(b_scales.data_ptr());
    g.bias = op.dense_as<float>("bias", bias, at::kFloat, {g.n});
    g.y = out->data_ptr();
    if (out != &made)
        op.apart("out", rows_of(*out, g.n * int64_t(out->element_size())),
                 {{"a", rows_of(a, g.k)}, {"b", rows_of(b, g.k)}, {"a_scales", numbers_of(a_scales)}, {"b_scales", numbers_of(b_scales)}, {"bias", block_of(bias)}});
    op.run(g_matmul, g);
    if (out != &made) written(*out);
    PyObject *result = in.args[6] == Py_None ? THPVariable_Wrap(*out) : Py_NewRef(in.args[6]);
    if (!result) throw python_error();
    return result;
}

PyObject *rms_norm(const Args &in)          // name, x, weight, residual, new_residual, eps, out, scales
{
    const char *name = PyUnicode_AsUTF8(in.args[0]);
    if (!name) throw python_error();
    const bool quantized = name[8] != 0;        // rms_norm_quantized
    const at::Tensor &x = in.tensor(1), &weight = in.tensor(2);
    const at::Tensor *residual = in.optional(3), *kept = in.optional(4), *out = in.optional(6), *scales = in.optional(7);
    if (x.dim() != 2) refuse(XL_E_SHAPE, name, ": x is [rows, k]");
    const Op op(name, x);
    const at::ScalarType type = x.scalar_type(), sum_type = residual ? residual->scalar_type() : kept ? kept->scalar_type() : type;
    xl_rms_norm_args a = {};
    a.dtype = type_code(name, "x", type);
    a.residual_dtype = type_code(name, "residual", sum_type);
    a.quantized = quantized;
    a.rows = x.size(0);
    a.k = x.size(1);
    a.eps = in.number(5);
    const int64_t blocks[] = {a.rows, (a.k + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK}, wide = (a.k + 15) / 16 * 16;
    const at::ScalarType out_type = quantized ? at::kFloat8_e4m3fn : type;
    at::Tensor made, made_scales, made_kept;
    if (!out) {
        made = op.make({a.rows, quantized ? wide : a.k}, out_type);
        if (quantized && wide != a.k) made.unsafeGetTensorImpl()->set_sizes_and_strides(x.sizes(), at::IntArrayRef{wide, 1});
        out = &made;
    }
    if (quantized && !scales) {     // a column for each block, as the quantiser leaves them
        const int64_t step[] = {1, a.rows};
        scales = &(made_scales = op.make(blocks, step, at::kFloat));
    }
    if (residual && !kept) kept = &(made_kept = op.make(x.sizes(), sum_type));
    op.check("x", x, type, x.sizes());
    op.check("out", *out, out_type, x.sizes());
    if (residual) op.check("residual", *residual, sum_type, x.sizes());
    if (kept) op.check("new_residual", *kept, sum_type, x.sizes());
    if (quantized) op.check("scales", *scales, at::kFloat, blocks);
    if (a.k > 1 && (x.stride(1) != 1 || out->stride(1) != 1 || (residual && residual->stride(1) != 1) || (kept && kept->stride(1) != 1)))
        refuse(XL_E_SHAPE, name, ": rows of x, out and the residuals must be contiguous");
    if (quantized) {
        check_readable(op, "out", *out);
        a.scale_row = scales->stride(0);
        a.scale_block = scales->stride(1);
        a.scales = static_cast<float *>(scales->data_ptr());
    }
    a.x_row = x.stride(0);
    a.y_row = out->stride(0);
    a.x = x.data_ptr();
    a.weight = op.dense_as<float>("weight", &weight, at::kFloat, {a.k});
    a.y = out->data_ptr();
    if (residual) {
        a.residual_row = residual->stride(0);
        a.residual = residual->data_ptr();
    }
    if (kept) {
        a.new_residual_row = kept->stride(0);
        a.new_residual = kept->data_ptr();
    }
    if (out != &made || (kept && kept != &made_kept) || (quantized && scales != &made_scales)) {
        const auto span = [&](const at::Tensor *t) { return t ? rows_of(*t, a.k * int64_t(t->element_size())) : xls::Span{}; };
        const Named factor = {"weight", block_of(&weight)}, sum = {"new_residual", span(kept)}, numbers = {"scales", quantized ? numbers_of(*scales) : xls::Span{}};
        Named input = {"x (or is it, as a whole)", span(&x)}, old = {"residual (or is it, as a whole)", span(residual)};
        if (quantized && scales != &made_scales) op.apart("scales", numbers.span, {{"x", input.span}, {"residual", old.span}, sum, factor});
        if (kept && kept != &made_kept) op.apart("new_residual", sum.span, {{"x", input.span}, {old.what, old.span == sum.span ? xls::Span{} : old.span}, factor});
        if (out != &made) {
            const xls::Span y = quantized ? rows_of(*out, wide) : span(out);
            if (!quantized && y == input.span) input.span = {};
            op.apart("out", y, {input, {"residual", old.span}, sum, factor, numbers});
        }
    }
    op.run(g_norm, a);
    if (out != &made) written(*out);
    if (quantized && scales != &made_scales) written(*scales);
    if (kept && kept != &made_kept) written(*kept);
    PyObject *parts[] = {result(in.args[6], *out), quantized ? result(in.args[7], *scales) : nullptr, kept ? result(in.args[4], *kept) : Py_NewRef(in.args[1])};
    PyObject *all = !parts[0] || (quantized && !parts[1]) || !parts[2] ? nullptr : quantized ? PyTuple_Pack(3, parts[0], parts[1], parts[2]) : PyTuple_Pack(2, parts[0], parts[2]);
    for (PyObject *p : parts) Py_XDECREF(p);
    if (!all) throw python_error();
    return all;
}

PyObject *add_adapters(const Args &in)      // y, x, down, up, index, scales, lengths, out
{
    const at::Tensor &y = in.tensor(0), &x = in.tensor(1), &down = in.tensor(2), &up = in.tensor(3), &index = in.tensor(4);
    const at::Tensor *scales = in.optional(5), *lengths = in.optional(6), *out = in.optional(7);
    if (y.dim() != 3 || x.dim() != 3 || down.dim() != 3) refuse(XL_E_SHAPE, "add_adapters: y is [batch, length, n], x [batch, length, k] and down [adapters, rank, k]");
    const Op op("add_adapters", y);
    const at::ScalarType type = y.scalar_type();
    xl_adapters_args a = {};
    a.dtype = type_code(op.name, "y", type);
    a.batch = y.size(0);
    a.length = y.size(1);
    a.n = y.size(2);
    a.k = x.size(2);
    a.adapters = down.size(0);
    a.rank = down.size(1);
    at::Tensor made;
    if (!out) out = &(made = op.make(y.sizes(), type));
    int64_t b, t;
    op.rows("y", y, type, y.sizes(), b, t);
    a.y_batch = b, a.y_token = t;
    op.rows("x", x, type, {a.batch, a.length, a.k}, b, t);
    a.x_batch = b, a.x_token = t;
    op.rows("out", *out, type, y.sizes(), b, t);
    a.out_batch = b, a.out_token = t;
    a.y = y.data_ptr();
    a.x = x.data_ptr();
    a.out = out->data_ptr();
    a.down = op.dense("down", &down, type, {a.adapters, a.rank, a.k});
    a.up = op.dense("up", &up, type, {a.adapters, a.n, a.rank});
    a.index = op.dense_as<int>("index", &index, at::kInt, {a.batch});
    a.scales = op.dense_as<float>("scales", scales, at::kFloat, {a.adapters});
    a.lengths = op.dense_as<int>("lengths", lengths, at::kInt, {a.batch});
    if (out != &made) {
        const xls::Span to = rows_of(*out), from = rows_of(y);
        op.apart("out", to, {{"y (or is it, as a whole)", from == to ? xls::Span{} : from}, {"x", rows_of(x)}, {"down", block_of(&down)}, {"up", block_of(&up)},
                             {"index", block_of(&index)}, {"scales", block_of(scales)}, {"lengths", block_of(lengths)}});
    }
    at::Tensor workspace;
    a.workspace_bytes = g_adapters_workspace(&a);
    if (a.workspace_bytes > 0) a.workspace = (workspace = op.make({a.workspace_bytes}, at::kByte)).data_ptr();
    op.run(g_adapters, a);
    if (out != &made) written(*out);
    PyObject *given = result(in.args[7], *out);
    if (!given) throw python_error();
    return given;
}

PyObject *gated_delta_rule(const Args &in)  // q, k, v, g, beta, scale, normalize, state, new_state, lengths, slots, out
{
    const at::Tensor &q = in.tensor(0), &k = in.tensor(1), &v = in.tensor(2), &g = in.tensor(3), &beta = in.tensor(4);
    const at::Tensor *state = in.optional(7), *lengths = in.optional(9), *slots = in.optional(10), *given = in.optional(11);
    if (q.dim() != 4 || v.dim() != 4) refuse(XL_E_SHAPE, "gated_delta_rule: q is [batch, length, key heads, dk] and v [batch, length, heads, dv]");
    const Op op("gated_delta_rule", v);
    const at::ScalarType type = v.scalar_type();
    xl_delta_args a = {};
    a.dtype = type_code(op.name, "v", type);
    a.batch = v.size(0);
    a.length = v.size(1);
    a.heads = v.size(2);
    a.dv = v.size(3);
    a.key_heads = q.size(2);
    a.dk = q.size(3);
    a.normalize = in.flag(6);
    const at::Tensor *kept = state_out(op, state, in.optional(8), slots);
    a.nslots = slots && state->dim() ? state->size(0) : a.batch;
    const int64_t shape[] = {a.nslots, a.heads, a.dk, a.dv}, keys[] = {a.batch, a.length, a.key_heads, a.dk}, tokens[] = {a.batch, a.length, a.heads};
    at::Tensor made, made_state;
    if (!given) given = &(made = op.make(v.sizes(), type));
    if (!kept) kept = &(made_state = op.make(shape, at::kFloat));
    int64_t b, t;
    op.heads("q", q, type, keys, a.q_batch, a.q_token, a.q_head);
    op.heads("k", k, type, keys, a.k_batch, a.k_token, a.k_head);
    op.heads("v", v, type, v.sizes(), a.v_batch, a.v_token, a.v_head);
    op.heads("out", *given, type, v.sizes(), a.y_batch, a.y_token, a.y_head);
    if (a.heads > 1 && a.dv > 0 && a.y_head != a.dv) refuse(XL_E_SHAPE, "gated_delta_rule: the heads of out must lie next to each other");
    op.rows("g", g, at::kFloat, tokens, b, t);
    a.g_batch = b, a.g_token = t;
    op.rows("beta", beta, at::kFloat, tokens, b, t);
    a.beta_batch = b, a.beta_token = t;
    a.scale = in.args[5] == Py_None ? 1. / std::sqrt(double(a.dk > 0 ? a.dk : 1)) : in.number(5);
    a.q = q.data_ptr();
    a.k = k.data_ptr();
    a.v = v.data_ptr();
    a.g = static_cast<const float *>(g.data_ptr());
    a.beta = static_cast<const float *>(beta.data_ptr());
    a.state = op.dense_as<float>("state", state, at::kFloat, shape);
    a.new_state = op.dense_as<float>("new_state", kept, at::kFloat, shape);
    a.lengths = op.dense_as<int>("lengths", lengths, at::kInt, {a.batch});
    a.slots = op.dense_as<int>("slots", slots, at::kInt, {a.batch});
    a.y = given->data_ptr();
    if (given != &made || kept != &made_state) {
        const Named old = {"state (or is it, as a whole)", a.state != a.new_state ? block_of(state) : xls::Span{}};
        const Named in_q = {"q", heads_of(q)}, in_k = {"k", heads_of(k)}, in_v = {"v", heads_of(v)}, in_g = {"g", rows_of(g)}, in_beta = {"beta", rows_of(beta)},
                    in_lengths = {"lengths", block_of(lengths)}, in_slots = {"slots", block_of(slots)};
        if (given != &made) op.apart("out", heads_of(*given), {in_q, in_k, in_v, in_g, in_beta, old, {"new_state", block_of(kept)}, in_lengths, in_slots});
        if (kept != &made_state) op.apart("new_state", block_of(kept), {in_q, in_k, in_v, in_g, in_beta, old, in_lengths, in_slots});
    }
    at::Tensor workspace;
    a.workspace_bytes = g_delta_workspace(&a);
    if (a.workspace_bytes > 0) a.workspace = (workspace = op.make({a.workspace_bytes}, at::kByte)).data_ptr();
    op.run(g_delta, a);
    if (given != &made) written(*given);
    if (kept != &made_state) written(*kept);
    return pair(in.args[11], *given, in.args[8] == Py_None && slots ? in.args[7] : in.args[8], *kept);
}

template <PyObject *(*F)(const Args &), int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N || !g_error) {
        PyErr_Format(PyExc_TypeError, "%d arguments wanted, %zd given, or not bound to a library", N, n);
        return nullptr;
    }
    try {
        return F(Args{args});
    } catch (const Refused &r) {
        return raised(r);
    }
    END_HANDLE_TH_ERRORS
}

// bind(address ..., exception): the library's functions, in the order of seq.py's list
PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long f[11];
    PyObject *error;
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &f[8], &f[9], &f[10], &error)) return nullptr;
    int i = 0;
    const auto set = [&](auto &function) { function = reinterpret_cast<std::decay_t<decltype(function)>>(f[i++]); };
    set(g_conv);
    set(g_scan);
    set(g_scan_workspace);
    set(g_quantize);
    set(g_matmul);
    set(g_norm);
    set(g_adapters);
    set(g_adapters_workspace);
    set(g_delta);
    set(g_delta_workspace);
    set(g_last_error);
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    Py_RETURN_NONE;
}

template <PyObject *(*F)(const Args &), int N> PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F, N>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<causal_conv, 9>("causal_conv"), method<selective_scan, 14>("selective_scan"), method<quantize, 5>("quantize"),
                         method<block_matmul, 7>("block_matmul"), method<rms_norm, 8>("rms_norm"), method<add_adapters, 8>("add_adapters"),
                         method<gated_delta_rule, 12>("gated_delta_rule"), {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_xl_seq", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__xl_seq(void) { return PyModule_Create(&module); }
