// xred_torch.cpp -- marshalling of torch tensors into the xred_* C ABI.
//
// A small call's kernel takes 2-3 us; checking and collecting its tensors one
// attribute at a time from Python took 6-30 us, and 1.1 ms for a batch of 256
// items of 8 sources.  These functions make the same checks on the tensors
// themselves and call the library with the interpreter lock released
// (allreduce of 8 x 8 KiB bf16 11.0 -> 4.0 us a call, that batch 1209 -> 97 us).
//
// Each returns the call's xred_status, or None, with nothing done, for
// anything but plain torch.Tensor / Parameter arguments that pass every check:
// the binding's Python code then handles the call, or raises its error.  No
// argument is kept, no result of a check is remembered.
#include <Python.h>

#include <ATen/Functions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstring>
#include <exception>
#include <vector>

#include "../../include/xred.h"

namespace {

// The library's entry points (addresses handed over by bind()) and torch's
// function that gives the current stream of a device.
decltype(&xred_allreduce_local) f_allreduce;
decltype(&xred_reduce_scatter_local) f_scatter;
decltype(&xred_reduce_copy_step) f_step;
decltype(&xred_acc_cast) f_cast;
decltype(&xred_batched_reduce) f_batched;
decltype(&xred_ring_reduce) f_ring;
decltype(&xred_allreduce_sim) f_sim;
decltype(&xred_fold_norm) f_fold_norm;
decltype(&xred_fold_norm_grad) f_fold_norm_grad;
decltype(&xred_fold_norm_grad_workspace) f_fold_norm_grad_workspace;
decltype(&xred_route) f_route;
decltype(&xred_route_grad) f_route_grad;
decltype(&xred_dispatch_plan) f_dispatch_plan;
decltype(&xred_dispatch_plan_workspace) f_dispatch_plan_workspace;
decltype(&xred_dispatch) f_dispatch;
decltype(&xred_combine) f_combine;
decltype(&xred_combine_grad) f_combine_grad;
decltype(&xred_group_product) f_group_product;
decltype(&xred_group_product_grad) f_group_product_grad;
decltype(&xred_gate) f_gate;
decltype(&xred_gate_grad) f_gate_grad;
decltype(&xred_quant_mx4) f_quant_mx4;
decltype(&xred_dequant_mx4) f_dequant_mx4;
PyObject *current_raw_stream;

// Raised to leave a call to the Python code.
struct Decline {};

struct Type {
    xred_dtype code;
    size_t size, acc;
};

bool text_is(PyObject *o, const char *s)
{
    return PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, s) == 0;
}

Type type_named(PyObject *name)
{
    static const struct {
        const char *name;
        Type t;
    } table[] = {
        {"f32", {XRED_FLOAT32, 4, 4}}, {"bf16", {XRED_BFLOAT16, 2, 4}},
        {"f16", {XRED_FLOAT16, 2, 4}}, {"i32", {XRED_INT32, 4, 4}},
        {"u32", {XRED_UINT32, 4, 4}}, {"i64", {XRED_INT64, 8, 8}},
        {"u64", {XRED_UINT64, 8, 8}}, {"e4m3", {XRED_FP8_E4M3, 1, 4}},
        {"e5m2", {XRED_FP8_E5M2, 1, 4}}, {"f64", {XRED_FLOAT64, 8, 8}},
        {"i8", {XRED_INT8, 1, 4}}, {"u8", {XRED_UINT8, 1, 4}}};
    for (const auto &e : table)
        if (text_is(name, e.name)) return e.t;
    throw Decline{};
}

Type type_of(const at::Tensor &t, PyObject *name)
{
    if (name != Py_None) return type_named(name);
    switch (t.scalar_type()) {
    case at::kFloat: return {XRED_FLOAT32, 4, 4};
    case at::kBFloat16: return {XRED_BFLOAT16, 2, 4};
    case at::kHalf: return {XRED_FLOAT16, 2, 4};
    case at::kInt: return {XRED_INT32, 4, 4};
    case at::kUInt32: return {XRED_UINT32, 4, 4};
    case at::kLong: return {XRED_INT64, 8, 8};
    case at::kUInt64: return {XRED_UINT64, 8, 8};
    case at::kFloat8_e4m3fn: return {XRED_FP8_E4M3, 1, 4};
    case at::kFloat8_e5m2: return {XRED_FP8_E5M2, 1, 4};
    case at::kDouble: return {XRED_FLOAT64, 8, 8};
    case at::kChar: return {XRED_INT8, 1, 4};
    case at::kByte: return {XRED_UINT8, 1, 4};
    default: throw Decline{};
    }
}

xred_op op_named(PyObject *o)
{
    if (text_is(o, "sum")) return XRED_SUM;
    if (text_is(o, "avg")) return XRED_AVG;
    if (text_is(o, "max")) return XRED_MAX;
    if (text_is(o, "min")) return XRED_MIN;
    if (text_is(o, "prod")) return XRED_PROD;
    throw Decline{};
}

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) throw Decline{};
    return THPVariable_Unpack(o);
}

// The data pointer of a contiguous tensor of n elements of `size` bytes on dev.
void *data_of(const at::Tensor &t, c10::Device dev, int64_t n, size_t size)
{
    if (!t.is_cuda() || t.device() != dev || !t.is_contiguous() ||
        t.element_size() != (int64_t)size || t.numel() != n)
        throw Decline{};
    return t.data_ptr();
}

// Flags or a status word: the same, or pinned host memory, of at least n words.
void *words_of(PyObject *o, c10::Device dev, int64_t n)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (t.is_cuda() ? t.device() != dev : !t.is_pinned()) throw Decline{};
    if (!t.is_contiguous() || t.element_size() != 4 || t.numel() < n) throw Decline{};
    return t.data_ptr();
}

// A list or tuple of 1..XRED_MAX_SRC tensors.
struct Sources {
    void *p[XRED_MAX_SRC];
    int n;
    Sources(PyObject *seq, c10::Device dev, int64_t numel, size_t size)
    {
        if (!PyList_CheckExact(seq) && !PyTuple_CheckExact(seq)) throw Decline{};
        const Py_ssize_t len = PySequence_Fast_GET_SIZE(seq);
        if (len < 1 || len > XRED_MAX_SRC) throw Decline{};
        n = (int)len;
        PyObject **o = PySequence_Fast_ITEMS(seq);
        for (int i = 0; i < n; ++i) p[i] = data_of(tensor(o[i]), dev, numel, size);
    }
};

// The stream argument: None (the device's current stream), a stream object or a handle.
void *stream_of(PyObject *o, c10::Device dev)
{
    PyObject *h;
    if (o == Py_None) {
        PyObject *index = PyLong_FromLong(dev.index());
        h = index ? PyObject_CallOneArg(current_raw_stream, index) : nullptr;
        Py_XDECREF(index);
    } else if (PyLong_CheckExact(o)) {
        h = o;
        Py_INCREF(h);
    } else {
        h = PyObject_GetAttrString(o, "cuda_stream");
    }
    void *s = h ? PyLong_AsVoidPtr(h) : nullptr;
    Py_XDECREF(h);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw Decline{};
    }
    return s;
}

template <class F>
int unlocked(F &&call)
{
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = (int)call();
    Py_END_ALLOW_THREADS
    return st;
}

// The body of every function: `want` arguments; f() gives a status, and
// whatever it throws leaves the call to the Python code.
template <class F>
PyObject *entry(Py_ssize_t nargs, Py_ssize_t want, F &&f)
{
    if (nargs != want || f_allreduce == nullptr) Py_RETURN_NONE;
    try {
        return PyLong_FromLong(f());
    } catch (const Decline &) {
    } catch (const std::exception &) {
    }
    Py_RETURN_NONE;
}

// allreduce(srcs, out, op, dtype, stream)
PyObject *allreduce(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 5, [&] {
        const at::Tensor &out = tensor(a[1]);
        const c10::Device dev = out.device();
        const Type t = type_of(out, a[3]);
        const int64_t n = out.numel();
        void *dst = data_of(out, dev, n, t.size);
        const Sources s(a[0], dev, n, t.size);
        const xred_op op = op_named(a[2]);
        void *stream = stream_of(a[4], dev);
        return unlocked([&] { return f_allreduce(s.p, s.n, dst, (size_t)n, t.code, op, stream); });
    });
}

// scatter(srcs, rank, out, op, dtype, stream)
PyObject *scatter(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 6, [&] {
        const at::Tensor &out = tensor(a[2]);
        const c10::Device dev = out.device();
        const Type t = type_of(out, a[4]);
        const int64_t n = out.numel();
        void *dst = data_of(out, dev, n, t.size);
        if (!PyList_CheckExact(a[0]) && !PyTuple_CheckExact(a[0])) throw Decline{};
        if (!PyLong_CheckExact(a[1])) throw Decline{};
        int over = 0;
        const long rank = PyLong_AsLongAndOverflow(a[1], &over);
        if (over || rank != (int)rank) throw Decline{};
        const Sources s(a[0], dev, n * (int64_t)PySequence_Fast_GET_SIZE(a[0]), t.size);
        const xred_op op = op_named(a[3]);
        void *stream = stream_of(a[5], dev);
        return unlocked([&] {
            return f_scatter(s.p, s.n, (int)rank, dst, (size_t)n, t.code, op, stream);
        });
    });
}

// step(in, acc, out, op, flags, dtype, stream)
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 7, [&] {
        const at::Tensor &in = tensor(a[0]);
        const c10::Device dev = in.device();
        const Type t = type_of(in, a[5]);
        const int64_t n = in.numel();
        const unsigned flags = (unsigned)PyLong_AsUnsignedLong(a[4]);
        void *src = data_of(in, dev, n, t.size), *acc = nullptr, *dst = nullptr;
        // what the flags do not use is passed on unchecked, as the library takes it
        if (flags != (XRED_STEP_INIT | XRED_STEP_FINAL))
            acc = data_of(tensor(a[1]), dev, n, t.acc);
        else if (a[1] != Py_None)
            acc = tensor(a[1]).data_ptr();
        if (flags & XRED_STEP_FINAL) dst = data_of(tensor(a[2]), dev, n, t.size);
        else if (a[2] != Py_None) dst = tensor(a[2]).data_ptr();
        const xred_op op = op_named(a[3]);
        void *stream = stream_of(a[6], dev);
        return unlocked([&] { return f_step(src, acc, dst, (size_t)n, t.code, op, flags, stream); });
    });
}

// cast(acc, out, dtype, stream)
PyObject *cast(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 4, [&] {
        const at::Tensor &out = tensor(a[1]);
        const c10::Device dev = out.device();
        const Type t = type_of(out, a[2]);
        const int64_t n = out.numel();
        void *dst = data_of(out, dev, n, t.size);
        void *acc = data_of(tensor(a[0]), dev, n, t.acc);
        void *stream = stream_of(a[3], dev);
        return unlocked([&] { return f_cast(acc, dst, (size_t)n, t.code, stream); });
    });
}

// batched(items, op, dtype, stream): a list of (sources, out) pairs
PyObject *batched(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 4, [&] {
        if (!PyList_CheckExact(a[0]) || PyList_GET_SIZE(a[0]) < 1) throw Decline{};
        const Type t = type_named(a[2]);
        const xred_op op = op_named(a[1]);
        const Py_ssize_t k = PyList_GET_SIZE(a[0]);
        if (k != (int)k) throw Decline{};
        std::vector<xred_item> items((size_t)k);
        std::vector<void *> ptrs;
        ptrs.reserve((size_t)k * 8);
        std::vector<size_t> first((size_t)k);
        c10::Device dev(c10::kCPU);
        for (Py_ssize_t i = 0; i < k; ++i) {
            PyObject *pair = PyList_GET_ITEM(a[0], i);
            if (!PyTuple_CheckExact(pair) || PyTuple_GET_SIZE(pair) != 2) throw Decline{};
            const at::Tensor &out = tensor(PyTuple_GET_ITEM(pair, 1));
            if (i == 0) dev = out.device();
            const int64_t n = out.numel();
            items[i].dst = data_of(out, dev, n, t.size);
            const Sources s(PyTuple_GET_ITEM(pair, 0), dev, n, t.size);
            first[i] = ptrs.size();
            ptrs.insert(ptrs.end(), s.p, s.p + s.n);
            items[i].count = (uint64_t)n;
            items[i].nsrc = (uint32_t)s.n;
            items[i].reserved = 0;
        }
        for (Py_ssize_t i = 0; i < k; ++i) items[i].srcs = ptrs.data() + first[i];
        void *stream = stream_of(a[3], dev);
        return unlocked([&] { return f_batched(items.data(), (int)k, t.code, op, 0, stream); });
    });
}

// ring(chunks, out, op, ready, epoch, timeout_us, status, dtype, stream)
PyObject *ring(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 9, [&] {
        const at::Tensor &out = tensor(a[1]);
        const c10::Device dev = out.device();
        const Type t = type_of(out, a[7]);
        const int64_t n = out.numel();
        void *dst = data_of(out, dev, n, t.size);
        const Sources s(a[0], dev, n, t.size);
        const xred_op op = op_named(a[2]);
        const uint32_t *ready = (const uint32_t *)words_of(a[3], dev, s.n);
        uint32_t *status = (uint32_t *)words_of(a[6], dev, 1);
        const unsigned long epoch = PyLong_AsUnsignedLongMask(a[4]);
        const unsigned long long timeout = PyLong_AsUnsignedLongLongMask(a[5]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            throw Decline{};
        }
        void *stream = stream_of(a[8], dev);
        return unlocked([&] {
            return f_ring(s.p, s.n, dst, (size_t)n, t.code, op, ready, (uint32_t)epoch, timeout,
                          status, stream);
        });
    });
}

// sim(sends, recvs, op, schedule, dtype, stream)
PyObject *sim(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 6, [&] {
        if ((!PyList_CheckExact(a[1]) && !PyTuple_CheckExact(a[1])) ||
            PySequence_Fast_GET_SIZE(a[1]) < 1)
            throw Decline{};
        const at::Tensor &out = tensor(PySequence_Fast_ITEMS(a[1])[0]);
        const c10::Device dev = out.device();
        const Type t = type_of(out, a[4]);
        const int64_t n = out.numel();
        const Sources recvs(a[1], dev, n, t.size), sends(a[0], dev, n, t.size);
        if (sends.n != recvs.n) throw Decline{};
        const xred_op op = op_named(a[2]);
        xred_schedule schedule;
        if (text_is(a[3], "ring")) schedule = XRED_SCHEDULE_RING;
        else if (text_is(a[3], "rhd")) schedule = XRED_SCHEDULE_RHD;
        else if (text_is(a[3], "ring1")) schedule = XRED_SCHEDULE_RING_ONE_LAUNCH;
        else if (text_is(a[3], "rhd1")) schedule = XRED_SCHEDULE_RHD_ONE_LAUNCH;
        else throw Decline{};
        void *stream = stream_of(a[5], dev);
        return unlocked([&] {
            return f_sim(sends.p, recvs.p, sends.n, (size_t)n, t.code, op, schedule, stream);
        });
    });
}

// ------------------------------------------------ around a reduced activation --
// A matrix argument: a 2-D tensor of this shape, dtype and device whose rows are
// contiguous; None where it may be absent.
struct Matrix {
    c10::Device dev;
    int64_t rows, columns;
    at::ScalarType type;

    xred_rows operator()(PyObject *o) const { return (*this)(o, columns, type); }
    xred_rows operator()(PyObject *o, int64_t n, at::ScalarType t) const
    {
        return o == Py_None ? xred_rows{nullptr, 0} : of(tensor(o), n, t);
    }
    xred_rows of(const at::Tensor &m, int64_t n, at::ScalarType t) const
    {
        if (!m.is_cuda() || m.device() != dev || m.scalar_type() != t || m.dim() != 2 ||
            m.size(0) != rows || m.size(1) != n || (n > 1 && m.stride(1) != 1) ||
            (rows > 1 && m.stride(0) < n))
            throw Decline{};
        return {m.data_ptr(), (uint64_t)(rows > 1 ? m.stride(0) : n)};
    }
};

// The matrix that gives a call its shape, dtype (fp32, bf16 or fp16 unless
// `any`) and device.
Matrix lead(PyObject *o, xred_dtype *dtype, bool any = false)
{
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.dim() != 2) throw Decline{};
    if (!any && t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16 &&
        t.scalar_type() != at::kHalf)
        throw Decline{};
    *dtype = type_of(t, Py_None).code;
    return {t.device(), t.size(0), t.size(1), t.scalar_type()};
}

// A contiguous tensor of n elements of one dtype, or None: nullptr.
void *vector(PyObject *o, c10::Device dev, int64_t n, at::ScalarType type)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != type) throw Decline{};
    return data_of(t, dev, n, c10::elementSize(type));
}

// A contiguous tokens x topk tensor.
void *slots(PyObject *o, c10::Device dev, int64_t tokens, int64_t topk, at::ScalarType type)
{
    const at::Tensor &t = tensor(o);
    if (t.dim() != 2 || t.size(0) != tokens || t.size(1) != topk) throw Decline{};
    return vector(o, dev, tokens * topk, type);
}

int64_t slots_per_token(PyObject *o)
{
    const at::Tensor &t = tensor(o);
    if (t.dim() != 2) throw Decline{};
    return t.size(1);
}

// Row weights in the call's dtype or fp32, or None.
const void *row_weights(PyObject *o, const Matrix &m, xred_dtype dtype, xred_dtype *type)
{
    *type = dtype;
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != m.type && t.scalar_type() != at::kFloat) throw Decline{};
    *type = t.scalar_type() == m.type ? dtype : XRED_FLOAT32;
    return data_of(t, m.dev, m.columns, t.element_size());
}

uint32_t u32_of(PyObject *o)
{
    if (!PyLong_CheckExact(o)) throw Decline{};
    int over = 0;
    const long x = PyLong_AsLongAndOverflow(o, &over);
    if (over || x < 0 || x > INT32_MAX) throw Decline{};
    return (uint32_t)x;
}

float float_of(PyObject *o)
{
    if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
    if (!PyLong_CheckExact(o)) throw Decline{};
    const double x = PyLong_AsDouble(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw Decline{};
    }
    return (float)x;
}

xred_score score_of(PyObject *o)
{
    if (text_is(o, "softmax")) return XRED_SCORE_SOFTMAX;
    if (text_is(o, "sigmoid")) return XRED_SCORE_SIGMOID;
    throw Decline{};
}

// The caller's workspace, or one from torch's allocator into `keep`, which belongs
// to the current stream; on a stream that the caller names the Python code
// allocates it.
void *workspace_of(PyObject *o, c10::Device dev, uint64_t need, PyObject *stream,
                   uint64_t *bytes, at::Tensor *keep)
{
    *bytes = 0;
    if (need == 0) return nullptr;
    if (o == Py_None) {
        if (stream != Py_None) throw Decline{};
        *keep = at::empty({(int64_t)need}, at::TensorOptions().dtype(at::kByte).device(dev));
        *bytes = need;
        return keep->data_ptr();
    }
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.device() != dev || !t.is_contiguous()) throw Decline{};
    *bytes = (uint64_t)t.numel() * t.element_size();
    return t.data_ptr();
}

// fold_norm(srcs, out, residual, weight, sum, out8, scale, rstd, group, eps, stream)
PyObject *fold_norm(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 11, [&] {
        if (!PyList_CheckExact(a[0]) && !PyTuple_CheckExact(a[0])) throw Decline{};
        const Py_ssize_t nsrc = PySequence_Fast_GET_SIZE(a[0]);
        if (nsrc < 1 || nsrc > XRED_MAX_SRC) throw Decline{};
        PyObject **src = PySequence_Fast_ITEMS(a[0]);
        xred_fold_norm_args n{};
        const Matrix m = lead(src[0], &n.dtype);
        const void *ptrs[XRED_MAX_SRC];
        n.srcs = ptrs;
        n.nsrc = (uint32_t)nsrc;
        for (Py_ssize_t i = 0; i < nsrc; ++i) {
            const xred_rows s = m(src[i]);
            if (i != 0 && s.stride != n.src_stride) throw Decline{};
            n.src_stride = s.stride;
            ptrs[i] = s.data;
        }
        n.group = u32_of(a[8]);
        n.rows = (uint64_t)m.rows;
        n.hidden = (uint64_t)m.columns;
        n.residual = m(a[2]);
        n.sum = m(a[4]);
        n.out = m(a[1]);
        if (a[5] != Py_None) {
            const at::ScalarType t = tensor(a[5]).scalar_type();
            if (t != at::kFloat8_e4m3fn && t != at::kByte) throw Decline{};
            n.out8 = m(a[5], m.columns, t);
        }
        n.scale = m(a[6], n.group ? (m.columns + n.group - 1) / n.group : 1, at::kFloat);
        n.weight = row_weights(a[3], m, n.dtype, &n.weight_dtype);
        n.rstd = (float *)vector(a[7], m.dev, m.rows, at::kFloat);
        n.eps = float_of(a[9]);
        void *stream = stream_of(a[10], m.dev);
        return unlocked([&] { return f_fold_norm(&n, stream); });
    });
}

// fold_norm_grad(dout, sum, rstd, dx, weight, dsum, dweight, workspace, stream)
PyObject *fold_norm_grad(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 9, [&] {
        xred_fold_norm_grad_args n{};
        const Matrix m = lead(a[1], &n.dtype);
        n.rows = (uint64_t)m.rows;
        n.hidden = (uint64_t)m.columns;
        n.dout = m(a[0]);
        n.sum = m(a[1]);
        n.dsum = m(a[5]);
        n.dx = m(a[3]);
        n.weight = row_weights(a[4], m, n.dtype, &n.weight_dtype);
        n.rstd = (const float *)vector(a[2], m.dev, m.rows, at::kFloat);
        n.dweight = (float *)vector(a[6], m.dev, m.columns, at::kFloat);
        const uint64_t need = n.dweight ? f_fold_norm_grad_workspace(n.rows, n.hidden) : 0;
        at::Tensor keep;
        n.workspace = workspace_of(a[7], m.dev, need, a[8], &n.workspace_bytes, &keep);
        void *stream = stream_of(a[8], m.dev);
        return unlocked([&] { return f_fold_norm_grad(&n, stream); });
    });
}

// route(logits, ids, weights, score, bias, groups, group_topk, group_score, renorm, scale, stream)
PyObject *route(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 11, [&] {
        xred_route_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        const int64_t k = slots_per_token(a[1]);
        if (m.columns > XRED_MAX_EXPERTS || k > XRED_MAX_TOPK) throw Decline{};
        n.tokens = (uint64_t)m.rows;
        n.experts = (uint32_t)m.columns;
        n.topk = (uint32_t)k;
        n.groups = u32_of(a[5]);
        n.group_topk = u32_of(a[6]);
        n.group_score = u32_of(a[7]);
        n.flags = a[8] == Py_True ? XRED_ROUTE_RENORM : a[8] == Py_False ? 0u : throw Decline{};
        n.logits = m(a[0]);
        n.bias = (const float *)vector(a[4], m.dev, m.columns, at::kFloat);
        n.ids = (int32_t *)slots(a[1], m.dev, m.rows, k, at::kInt);
        n.weights = (float *)slots(a[2], m.dev, m.rows, k, at::kFloat);
        n.score = score_of(a[3]);
        n.scale = float_of(a[9]);
        void *stream = stream_of(a[10], m.dev);
        return unlocked([&] { return f_route(&n, stream); });
    });
}

// route_grad(logits, ids, dweights, dlogits, score, renorm, scale, stream)
PyObject *route_grad(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 8, [&] {
        xred_route_grad_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        const int64_t k = slots_per_token(a[1]);
        if (m.columns > XRED_MAX_EXPERTS || k > XRED_MAX_TOPK) throw Decline{};
        n.tokens = (uint64_t)m.rows;
        n.experts = (uint32_t)m.columns;
        n.topk = (uint32_t)k;
        n.flags = a[5] == Py_True ? XRED_ROUTE_RENORM : a[5] == Py_False ? 0u : throw Decline{};
        n.logits = m(a[0]);
        n.dlogits = m(a[3]);
        n.ids = (const int32_t *)slots(a[1], m.dev, m.rows, k, at::kInt);
        n.dweights = (const float *)slots(a[2], m.dev, m.rows, k, at::kFloat);
        n.score = score_of(a[4]);
        n.scale = float_of(a[6]);
        void *stream = stream_of(a[7], m.dev);
        return unlocked([&] { return f_route_grad(&n, stream); });
    });
}

// dispatch_plan(ids, counts, offsets, pos, slots, workspace, stream)
PyObject *dispatch_plan(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 7, [&] {
        const at::Tensor &ids = tensor(a[0]), &counts = tensor(a[1]);
        if (!ids.is_cuda() || ids.dim() != 2) throw Decline{};
        const c10::Device dev = ids.device();
        const int64_t tokens = ids.size(0), k = ids.size(1), experts = counts.numel();
        if (experts < 1 || experts > XRED_MAX_EXPERTS || k < 1 || k > XRED_MAX_TOPK) throw Decline{};
        xred_dispatch_plan_args n{};
        n.tokens = (uint64_t)tokens;
        n.experts = (uint32_t)experts;
        n.topk = (uint32_t)k;
        n.ids = (const int32_t *)slots(a[0], dev, tokens, k, at::kInt);
        n.counts = (int32_t *)vector(a[1], dev, experts, at::kInt);
        n.offsets = (int32_t *)vector(a[2], dev, experts + 1, at::kInt);
        n.pos = (int32_t *)slots(a[3], dev, tokens, k, at::kInt);
        n.slots = (int32_t *)vector(a[4], dev, tokens * k, at::kInt);
        at::Tensor keep;
        n.workspace = workspace_of(a[5], dev,
                                   f_dispatch_plan_workspace((uint64_t)(tokens * k), n.experts),
                                   a[6], &n.workspace_bytes, &keep);
        void *stream = stream_of(a[6], dev);
        return unlocked([&] { return f_dispatch_plan(&n, stream); });
    });
}

// dispatch(x, pos, out, scale, out_scale, stream)
PyObject *dispatch(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 6, [&] {
        xred_dispatch_args n{};
        const Matrix m = lead(a[0], &n.dtype, true);
        const int64_t k = slots_per_token(a[1]);
        if (k < 1 || k > XRED_MAX_TOPK || (a[3] == Py_None) != (a[4] == Py_None)) throw Decline{};
        const at::Tensor &out = tensor(a[2]);
        if (out.dim() != 2) throw Decline{};
        const Matrix to{m.dev, out.size(0), m.columns, m.type};
        n.tokens = (uint64_t)m.rows;
        n.hidden = (uint64_t)m.columns;
        n.out_rows = (uint64_t)to.rows;
        n.topk = (uint32_t)k;
        n.x = m(a[0]);
        n.out = to(a[2]);
        if (a[3] != Py_None) {
            const int64_t columns = slots_per_token(a[3]);
            n.scale_columns = (uint64_t)columns;
            n.scale = m(a[3], columns, at::kFloat);
            n.out_scale = to(a[4], columns, at::kFloat);
        }
        n.pos = (const int32_t *)slots(a[1], m.dev, m.rows, k, at::kInt);
        void *stream = stream_of(a[5], m.dev);
        return unlocked([&] { return f_dispatch(&n, stream); });
    });
}

// combine(y, pos, out, weights, base, stream)
PyObject *combine(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 6, [&] {
        xred_combine_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        const at::Tensor &pos = tensor(a[1]);
        const int64_t k = slots_per_token(a[1]);
        if (k < 1 || k > XRED_MAX_TOPK) throw Decline{};
        const Matrix to{m.dev, pos.size(0), m.columns, m.type};
        n.tokens = (uint64_t)to.rows;
        n.hidden = (uint64_t)m.columns;
        n.y_rows = (uint64_t)m.rows;
        n.topk = (uint32_t)k;
        n.y = m(a[0]);
        n.base = to(a[4]);
        if (a[2] == Py_None) throw Decline{};
        n.out = to(a[2]);
        n.pos = (const int32_t *)slots(a[1], m.dev, to.rows, k, at::kInt);
        if (a[3] != Py_None)
            n.weights = (const float *)slots(a[3], m.dev, to.rows, k, at::kFloat);
        void *stream = stream_of(a[5], m.dev);
        return unlocked([&] { return f_combine(&n, stream); });
    });
}

// combine_grad(dout, y, pos, weights, dy, dweights, stream)
PyObject *combine_grad(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 7, [&] {
        xred_combine_grad_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        const at::Tensor &dy = tensor(a[4]);
        const int64_t k = slots_per_token(a[2]);
        if (k < 1 || k > XRED_MAX_TOPK || dy.dim() != 2) throw Decline{};
        if (a[1] == Py_None && a[5] != Py_None) throw Decline{};
        const Matrix to{m.dev, dy.size(0), m.columns, m.type};
        n.tokens = (uint64_t)m.rows;
        n.hidden = (uint64_t)m.columns;
        n.y_rows = (uint64_t)to.rows;
        n.topk = (uint32_t)k;
        n.dout = m(a[0]);
        n.y = to(a[1]);
        n.dy = to(a[4]);
        n.pos = (const int32_t *)slots(a[2], m.dev, m.rows, k, at::kInt);
        n.weights = (const float *)slots(a[3], m.dev, m.rows, k, at::kFloat);
        if (a[5] != Py_None) n.dweights = (float *)slots(a[5], m.dev, m.rows, k, at::kFloat);
        void *stream = stream_of(a[6], m.dev);
        return unlocked([&] { return f_combine_grad(&n, stream); });
    });
}

// ------------------------------------------------ between dispatch and combine --
// The experts' matrices, each rows x columns: the first one, and the elements from one
// to the next.
xred_rows stack_of(PyObject *o, c10::Device dev, int64_t experts, int64_t rows, int64_t columns,
                   at::ScalarType type, uint64_t *apart)
{
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.device() != dev || t.scalar_type() != type || t.dim() != 3 ||
        t.size(0) != experts || t.size(1) != rows || t.size(2) != columns ||
        (columns > 1 && t.stride(2) != 1) || (rows > 1 && t.stride(1) < columns))
        throw Decline{};
    const int64_t stride = rows > 1 ? t.stride(1) : columns;
    *apart = (uint64_t)(experts > 1 ? t.stride(0) : rows * stride);
    return {t.data_ptr(), (uint64_t)stride};
}

const int32_t *offsets_of(PyObject *o, c10::Device dev, uint32_t *experts)
{
    const at::Tensor &t = tensor(o);
    if (t.dim() != 1 || t.numel() < 2 || t.numel() > XRED_MAX_EXPERTS + 1) throw Decline{};
    *experts = (uint32_t)t.numel() - 1;
    return (const int32_t *)vector(o, dev, t.numel(), at::kInt);
}

bool flag_of(PyObject *o)
{
    if (o != Py_True && o != Py_False) throw Decline{};
    return o == Py_True;
}

// An output's matrix of fp32, bf16 or fp16.
xred_rows typed_rows(PyObject *o, const Matrix &m, xred_dtype *dtype)
{
    const Matrix to = lead(o, dtype);
    if (to.dev != m.dev || to.rows != m.rows || to.columns != m.columns) throw Decline{};
    return m(o, m.columns, to.type);
}

// group_product(x, w, offsets, out, scale, w_scale, transpose, stream)
PyObject *group_product(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 8, [&] {
        xred_group_product_args n{};
        const Matrix m = lead(a[0], &n.dtype, true);
        const int64_t columns = slots_per_token(a[3]);
        const bool mx4 = n.dtype == XRED_UINT8, scaled = mx4 || n.dtype == XRED_FP8_E4M3;
        const bool across = flag_of(a[6]);
        if (!scaled && n.dtype != XRED_FLOAT32 && n.dtype != XRED_BFLOAT16 &&
            n.dtype != XRED_FLOAT16)
            throw Decline{};
        if (scaled != (a[4] != Py_None) || scaled != (a[5] != Py_None) || (mx4 && m.columns % 16))
            throw Decline{};
        n.rows = (uint64_t)m.rows;
        n.n = (uint64_t)columns;
        n.k = (uint64_t)(mx4 ? 2 * m.columns : m.columns);
        n.flags = (across ? XRED_PRODUCT_TRANSPOSE : 0u) | (mx4 ? XRED_PRODUCT_MX4 : 0u);
        n.offsets = offsets_of(a[2], m.dev, &n.experts);
        n.x = m(a[0]);
        n.out = typed_rows(a[3], Matrix{m.dev, m.rows, columns, m.type}, &n.out_dtype);
        if (!scaled && n.out_dtype != n.dtype && n.out_dtype != XRED_FLOAT32) throw Decline{};
        n.w = across ? stack_of(a[1], m.dev, n.experts, m.columns, columns, m.type, &n.w_expert)
                     : stack_of(a[1], m.dev, n.experts, columns, m.columns, m.type, &n.w_expert);
        if (scaled) {
            const at::ScalarType t = mx4 ? at::kByte : at::kFloat;
            const int64_t parts = mx4 ? m.columns / 16 : (m.columns + 127) / 128;
            n.scale = m(a[4], parts, t);
            n.w_scale = stack_of(a[5], m.dev, n.experts, mx4 ? columns : (columns + 127) / 128, parts,
                                 t, &n.w_scale_expert);
        }
        void *stream = stream_of(a[7], m.dev);
        return unlocked([&] { return f_group_product(&n, stream); });
    });
}

// group_product_grad(dout, x, offsets, dw, add, stream)
PyObject *group_product_grad(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 6, [&] {
        xred_group_product_grad_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        const int64_t k = slots_per_token(a[1]);
        n.rows = (uint64_t)m.rows;
        n.n = (uint64_t)m.columns;
        n.k = (uint64_t)k;
        n.flags = flag_of(a[4]) ? XRED_PRODUCT_ADD : 0u;
        n.offsets = offsets_of(a[2], m.dev, &n.experts);
        n.dout = m(a[0]);
        if (a[1] == Py_None) throw Decline{};
        n.x = m(a[1], k, m.type);
        const at::ScalarType to = tensor(a[3]).scalar_type();
        if (to != m.type && to != at::kFloat) throw Decline{};
        n.dw_dtype = to == m.type ? n.dtype : XRED_FLOAT32;
        n.dw = stack_of(a[3], m.dev, n.experts, m.columns, k, to, &n.dw_expert);
        void *stream = stream_of(a[5], m.dev);
        return unlocked([&] { return f_group_product_grad(&n, stream); });
    });
}

// The last of offsets, or None.
const int32_t *row_count(PyObject *o, c10::Device dev)
{
    if (o == Py_None) return nullptr;
    const int64_t n = tensor(o).numel();
    if (n < 1) throw Decline{};
    return (const int32_t *)vector(o, dev, n, at::kInt) + n - 1;
}

// gate(x, out, out8, scale, group, offsets, stream)
PyObject *gate(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 7, [&] {
        xred_gate_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        if (m.columns % 2) throw Decline{};
        const int64_t width = m.columns / 2;
        n.rows = (uint64_t)m.rows;
        n.width = (uint64_t)width;
        n.group = u32_of(a[4]);
        n.x = m(a[0]);
        n.out = m(a[1], width, m.type);
        if (a[2] != Py_None) {
            const at::ScalarType t = tensor(a[2]).scalar_type();
            if (t != at::kFloat8_e4m3fn && t != at::kByte) throw Decline{};
            n.out8 = m(a[2], width, t);
        }
        n.scale = m(a[3], n.group ? (width + n.group - 1) / n.group : 1, at::kFloat);
        n.count = row_count(a[5], m.dev);
        void *stream = stream_of(a[6], m.dev);
        return unlocked([&] { return f_gate(&n, stream); });
    });
}

// gate_grad(dout, x, dx, offsets, stream)
PyObject *gate_grad(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 5, [&] {
        xred_gate_grad_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        if (a[1] == Py_None || a[2] == Py_None) throw Decline{};
        n.rows = (uint64_t)m.rows;
        n.width = (uint64_t)m.columns;
        n.dout = m(a[0]);
        n.x = m(a[1], 2 * m.columns, m.type);
        n.dx = m(a[2], 2 * m.columns, m.type);
        n.count = row_count(a[3], m.dev);
        void *stream = stream_of(a[4], m.dev);
        return unlocked([&] { return f_gate_grad(&n, stream); });
    });
}

// quant_mx4(x, out4, scale, stream)
PyObject *quant_mx4(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 4, [&] {
        xred_quant_mx4_args n{};
        const Matrix m = lead(a[0], &n.dtype);
        if (a[1] == Py_None || a[2] == Py_None) throw Decline{};
        const int64_t blocks = (m.columns + 31) / 32;
        n.rows = (uint64_t)m.rows;
        n.columns = (uint64_t)m.columns;
        n.x = m(a[0]);
        n.out4 = m(a[1], 16 * blocks, at::kByte);
        n.scale = m(a[2], blocks, at::kByte);
        void *stream = stream_of(a[3], m.dev);
        return unlocked([&] { return f_quant_mx4(&n, stream); });
    });
}

// dequant_mx4(x4, scale, out, stream)
PyObject *dequant_mx4(PyObject *, PyObject *const *a, Py_ssize_t nargs)
{
    return entry(nargs, 4, [&] {
        xred_dequant_mx4_args n{};
        const Matrix m = lead(a[2], &n.dtype);
        if (a[0] == Py_None || a[1] == Py_None) throw Decline{};
        const int64_t blocks = (m.columns + 31) / 32;
        n.rows = (uint64_t)m.rows;
        n.columns = (uint64_t)m.columns;
        n.x4 = m(a[0], 16 * blocks, at::kByte);
        n.scale = m(a[1], blocks, at::kByte);
        n.out = m(a[2]);
        void *stream = stream_of(a[3], m.dev);
        return unlocked([&] { return f_dequant_mx4(&n, stream); });
    });
}

// bind(current_raw_stream, {name: address}): once, by the loader.
PyObject *bind(PyObject *, PyObject *args)
{
    PyObject *get, *addr;
    if (!PyArg_ParseTuple(args, "OO!", &get, &PyDict_Type, &addr)) return nullptr;
    auto take = [&](const char *name, auto &f) {
        PyObject *v = PyDict_GetItemString(addr, name);
        void *p = v ? PyLong_AsVoidPtr(v) : nullptr;
        f = (std::remove_reference_t<decltype(f)>)p;
        if (p == nullptr && !PyErr_Occurred())
            PyErr_Format(PyExc_ValueError, "no address for %s", name);
        return p != nullptr;
    };
    decltype(f_allreduce) all = nullptr;
    if (!take("xred_reduce_scatter_local", f_scatter) || !take("xred_reduce_copy_step", f_step) ||
        !take("xred_acc_cast", f_cast) || !take("xred_batched_reduce", f_batched) ||
        !take("xred_ring_reduce", f_ring) || !take("xred_allreduce_sim", f_sim) ||
        !take("xred_fold_norm", f_fold_norm) || !take("xred_fold_norm_grad", f_fold_norm_grad) ||
        !take("xred_fold_norm_grad_workspace", f_fold_norm_grad_workspace) ||
        !take("xred_route", f_route) || !take("xred_route_grad", f_route_grad) ||
        !take("xred_dispatch_plan", f_dispatch_plan) ||
        !take("xred_dispatch_plan_workspace", f_dispatch_plan_workspace) ||
        !take("xred_dispatch", f_dispatch) || !take("xred_combine", f_combine) ||
        !take("xred_combine_grad", f_combine_grad) ||
        !take("xred_group_product", f_group_product) ||
        !take("xred_group_product_grad", f_group_product_grad) || !take("xred_gate", f_gate) ||
        !take("xred_gate_grad", f_gate_grad) || !take("xred_quant_mx4", f_quant_mx4) ||
        !take("xred_dequant_mx4", f_dequant_mx4) ||
        !take("xred_allreduce_local", all))
        return nullptr;
    Py_INCREF(get);
    Py_XSETREF(current_raw_stream, get);
    f_allreduce = all;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"allreduce", (PyCFunction)(void *)allreduce, METH_FASTCALL, nullptr},
    {"scatter", (PyCFunction)(void *)scatter, METH_FASTCALL, nullptr},
    {"step", (PyCFunction)(void *)step, METH_FASTCALL, nullptr},
    {"cast", (PyCFunction)(void *)cast, METH_FASTCALL, nullptr},
    {"batched", (PyCFunction)(void *)batched, METH_FASTCALL, nullptr},
    {"ring", (PyCFunction)(void *)ring, METH_FASTCALL, nullptr},
    {"sim", (PyCFunction)(void *)sim, METH_FASTCALL, nullptr},
    {"fold_norm", (PyCFunction)(void *)fold_norm, METH_FASTCALL, nullptr},
    {"fold_norm_grad", (PyCFunction)(void *)fold_norm_grad, METH_FASTCALL, nullptr},
    {"route", (PyCFunction)(void *)route, METH_FASTCALL, nullptr},
    {"route_grad", (PyCFunction)(void *)route_grad, METH_FASTCALL, nullptr},
    {"dispatch_plan", (PyCFunction)(void *)dispatch_plan, METH_FASTCALL, nullptr},
    {"dispatch", (PyCFunction)(void *)dispatch, METH_FASTCALL, nullptr},
    {"combine", (PyCFunction)(void *)combine, METH_FASTCALL, nullptr},
    {"combine_grad", (PyCFunction)(void *)combine_grad, METH_FASTCALL, nullptr},
    {"group_product", (PyCFunction)(void *)group_product, METH_FASTCALL, nullptr},
    {"group_product_grad", (PyCFunction)(void *)group_product_grad, METH_FASTCALL, nullptr},
    {"gate", (PyCFunction)(void *)gate, METH_FASTCALL, nullptr},
    {"gate_grad", (PyCFunction)(void *)gate_grad, METH_FASTCALL, nullptr},
    {"quant_mx4", (PyCFunction)(void *)quant_mx4, METH_FASTCALL, nullptr},
    {"dequant_mx4", (PyCFunction)(void *)dequant_mx4, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_xred_torch",
                      "Marshalling of torch tensors into the xred_* C ABI.", -1, methods};

}  // namespace

#define XRED_TEXT_(x) #x
#define XRED_TEXT(x) XRED_TEXT_(x)

// `python` and `torch`: what the module was compiled against, for the loader.
PyMODINIT_FUNC PyInit__xred_torch()
{
    PyObject *m = PyModule_Create(&module);
    if (m != nullptr &&
        (PyModule_AddStringConstant(
             m, "python", XRED_TEXT(PY_MAJOR_VERSION) "." XRED_TEXT(PY_MINOR_VERSION)) < 0 ||
         PyModule_AddStringConstant(m, "torch",
                                    XRED_TEXT(TORCH_VERSION_MAJOR) "." XRED_TEXT(
                                        TORCH_VERSION_MINOR) "." XRED_TEXT(TORCH_VERSION_PATCH)) < 0)) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
