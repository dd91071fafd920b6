// Python entry points of include/experts_fp8.h in the module `_native`: argument checks, result tensors, stream and library
// call in one step; nothing here computes.
#include "py_args.h"

#include <vector>

#include <ATen/hip/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/util/SmallVector.h>

#include "../../include/experts_fp8.h"

extern PyMethodDef experts_methods[];
void experts_library(void *handle);

namespace {

using namespace c2py;

#define LIBRARY_CALLS(X)                                                                                                          \
    X(quantize_fp8_rows) X(quantize_fp8_columns) X(quantize_fp8_tiles) X(silu_gate_backward) X(gemm_fp8_nt) X(gemm_fp8_experts)   \
    X(gemm_fp8_experts_grad) X(route_experts) X(route_experts_backward) X(expert_rows) X(expert_rows_capacity) X(combine_experts) \
    X(combine_experts_backward)
struct Library {
#define CALL(name) decltype(&::name) name;
    LIBRARY_CALLS(CALL)
#undef CALL
} lib;
const char *missing = nullptr;   // one that the loaded library has not got (a library from before these calls)

template <class... A>
[[noreturn]] void refuse(PyObject *error, const char *format, A... a)
{
    PyErr_Format(error, format, a...);
    throw PyFail{};
}

// A call of the library, the interpreter lock given up for it (the arguments' checks are done by then).
template <class... P, class... A>
void run(const char *what, int (*call)(P...), A... a)
{
    int rc;
    {
        NoGil unlocked;
        rc = call(static_cast<P>(a)...);
    }
    check(rc, what);
}

int type_of(at::ScalarType t)   // -1: none of the three
{
    return t == at::kFloat ? EXPERTS_F32 : t == at::kBFloat16 ? EXPERTS_BF16 : t == at::kHalf ? EXPERTS_F16 : -1;
}
int type_of(const at::Tensor &t, const char *what)
{
    const int type = type_of(t.scalar_type());
    if (type < 0) refuse(PyExc_TypeError, "%s must be float32, bfloat16 or float16", what);
    return type;
}
int as_extent(int64_t n, const char *what)
{
    if (n > 0x7fffffff) refuse(PyExc_ValueError, "%s has an extent of 2^31 or more", what);
    return (int)n;
}

// A whole number (as_int takes them modulo 2^32, as its callers always have)
int whole(PyObject *o, const char *what)
{
    PyObject *i = PyNumber_Index(o);
    if (!i) throw PyFail{};
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(i, &over);
    Py_DECREF(i);
    if (over || v != (int)v) refuse(PyExc_ValueError, "%s is out of range", what);
    return (int)v;
}

// The call's device (the first tensor's, which must be the current one) and stream.  Results are allocated for the stream that the call runs on.
struct Call {
    int device;
    c10::hip::HIPStream stream;
    static int none_yet()
    {
        if (missing) refuse(PyExc_RuntimeError, "the loaded library has no symbol %s", missing);
        return -1;
    }
    explicit Call(PyObject *s) : device(none_yet()), stream(c10::hip::getCurrentHIPStream())
    {
        if (s == Py_None) return;
        PyObject *id = PyObject_GetAttrString(s, "stream_id"), *index = id ? PyObject_GetAttrString(s, "device_index") : nullptr;
        const bool got = index != nullptr;
        const int64_t id_ = got ? PyLong_AsLongLong(id) : 0, index_ = got ? PyLong_AsLongLong(index) : 0;
        Py_XDECREF(id);
        Py_XDECREF(index);
        if (!got || PyErr_Occurred()) throw PyFail{};
        // (torch's streams say "cuda" where HIP's own say "hip")
        stream = c10::hip::HIPStream::unpack3(id_, (c10::DeviceIndex)index_, c10::DeviceType::HIP);
    }
    const at::Tensor &on_device(const at::Tensor &t, const char *what)
    {
        if (!t.is_cuda()) refuse(PyExc_TypeError, "%s must be a CUDA tensor", what);
        // (a result that autograd knows nothing of must not stand in for one that it does)
        if (t.requires_grad() && c10::GradMode::is_enabled())
            refuse(PyExc_ValueError, "%s requires a gradient, which this call does not record: call it under torch.no_grad() or in an autograd.Function", what);
        if (device < 0) {
            device = t.get_device();
            if (device != stream.device_index()) refuse(PyExc_ValueError, "%s is on device %d, the stream on device %d", what, device, (int)stream.device_index());
        } else if (t.get_device() != device) {
            refuse(PyExc_ValueError, "%s is on device %d, not on device %d", what, (int)t.get_device(), device);
        }
        return t;
    }
    // a tensor whose last dimension is dense, of `dims` dimensions
    const at::Tensor &rows(PyObject *o, int dims, const char *what)
    {
        const at::Tensor &t = on_device(tensor(o, what), what);
        require_dims(t, dims, what);
        if (t.size(-1) > 1 && t.stride(-1) != 1) refuse(PyExc_ValueError, "%s must have rows of neighbouring elements", what);
        return t;
    }
    const at::Tensor &e4m3(PyObject *o, int dims, const char *what)
    {
        const at::Tensor &t = rows(o, dims, what);
        if (t.scalar_type() != at::kFloat8_e4m3fn) refuse(PyExc_TypeError, "%s must be float8_e4m3fn", what);
        return t;
    }
    const at::Tensor &dense(PyObject *o, at::ScalarType type, at::IntArrayRef shape, const char *what)
    {
        const at::Tensor &t = on_device(tensor(o, what), what);
        if (t.scalar_type() != type) refuse(PyExc_TypeError, "%s must be %s", what, type == at::kInt ? "int32" : "float32");
        if (!t.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous", what);
        if (t.sizes() != shape) refuse(PyExc_ValueError, "%s has another shape than the other arguments ask for", what);
        return t;
    }
    void *handle() const { return stream.stream(); }
};

// Distance of two rows: of a single row any distance will do.
int64_t row_distance(const at::Tensor &t, const char *what)
{
    const int64_t n = t.size(-1);
    if (t.size(-2) <= 1) return n > t.stride(-2) ? n : t.stride(-2);
    if (t.stride(-2) < n) refuse(PyExc_ValueError, "%s must not have rows that overlap", what);
    return t.stride(-2);
}

// Results, the caller's (a tensor, or a tuple of them) or new ones for the call's stream.
struct Results {
    Call &call;
    PyObject *given;
    c10::SmallVector<at::Tensor, 4> made;
    size_t count;
    Results(Call &c, PyObject *o, size_t n) : call(c), given(o == Py_None ? nullptr : o), count(n)
    {
        if (given && n > 1 && (!PyTuple_Check(given) || (size_t)PyTuple_GET_SIZE(given) != n)) refuse(PyExc_TypeError, "out must be a tuple of %d tensors", (int)n);
    }
    // the next result: [..., r, c] with rows `distance` apart if it is made here
    at::Tensor next(at::IntArrayRef shape, at::ScalarType type, int64_t distance, const at::Tensor &like, const char *what)
    {
        if (given) {
            const at::Tensor &t = call.on_device(tensor(count > 1 ? PyTuple_GET_ITEM(given, made.size()) : given, what), what);
            if (t.scalar_type() != type) refuse(PyExc_TypeError, "%s has another type than the result", what);
            if (t.sizes() != shape) refuse(PyExc_ValueError, "%s has another shape than the result", what);
            if (t.size(-1) > 1 && t.stride(-1) != 1) refuse(PyExc_ValueError, "%s must have rows of neighbouring elements", what);
            made.push_back(t);
        } else {
            const c10::hip::HIPStream now = c10::hip::getCurrentHIPStream();
            const bool other = now != call.stream;
            c10::SmallVector<int64_t, 4> strides(shape.size(), 1);
            if (shape.size() > 1) strides[shape.size() - 2] = distance ? distance : shape.back();
            for (int i = (int)shape.size() - 3; i >= 0; --i) strides[i] = strides[i + 1] * shape[i + 1];
            if (other) c10::hip::setCurrentHIPStream(call.stream);
            try {
                NoGil unlocked;
                made.push_back(at::detail::empty_strided_cuda(shape, strides, type, like.device()));   // (without the dispatcher: half the time)
            } catch (...) {
                if (other) c10::hip::setCurrentHIPStream(now);
                throw;
            }
            if (other) c10::hip::setCurrentHIPStream(now);
        }
        return made.back();
    }
    at::Tensor dense(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like, const char *what)
    {
        at::Tensor t = next(shape, type, 0, like, what);
        if (!t.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous", what);
        return t;
    }
    PyObject *result()
    {
        if (given) {
            Py_INCREF(given);
            return given;
        }
        if (count == 1) return THPVariable_Wrap(std::move(made[0]));
        PyObject *t = PyTuple_New((Py_ssize_t)count);
        if (!t) throw PyFail{};
        for (size_t i = 0; i < count; ++i) {
            PyObject *v = THPVariable_Wrap(std::move(made[i]));
            if (!v) {
                Py_DECREF(t);
                throw PyFail{};
            }
            PyTuple_SET_ITEM(t, (Py_ssize_t)i, v);
        }
        return t;
    }
};

int64_t blocks_of(int64_t n) { return (n + EXPERTS_BLOCK - 1) / EXPERTS_BLOCK; }
int64_t whole16(int64_t n) { return (n + 15) / 16 * 16; }   // rows of 8-bit results begin on 16 bytes

enum Form { ROWS, COLUMNS, BOTH, TILES, TILES_T };

// (x, form, gate, take, per_row, out, stream)
NATIVE(quantize_fp8, 7, {
    Call call(a[6]);
    const int form = as_int(a[1]);
    const bool tiles = form >= TILES;
    const int dims = tiles && tensor(a[0], "x").dim() == 3 ? 3 : 2;
    const at::Tensor &x = call.rows(a[0], dims, "x");
    const int type = type_of(x, "x"), gate = as_bool(a[2]), per_row = whole(a[4], "per_row");
    if (gate && tiles) refuse(PyExc_ValueError, "a gated activation has no form \"tiles\"");
    if (gate && x.size(-1) % 2) refuse(PyExc_ValueError, "x must have an even number of columns with a gate");
    const at::Tensor *take = nullptr;
    if (a[3] != Py_None) {
        if (tiles) refuse(PyExc_ValueError, "rows go with the forms \"rows\" and \"columns\"");
        take = &call.on_device(tensor(a[3], "rows"), "rows");
        if (take->scalar_type() != at::kInt || take->dim() != 1 || !take->is_contiguous()) refuse(PyExc_TypeError, "rows must be a contiguous int32 vector");
    }
    const int64_t ld = row_distance(x, "x");
    if (dims == 3 && x.size(0) > 1 && x.stride(0) != x.size(1) * ld) refuse(PyExc_ValueError, "the matrices of x must follow one another");
    const int64_t count = dims == 3 ? x.size(0) : 1;
    const int src_rows = as_extent(x.size(-2), "x"), rows = take ? as_extent(take->size(0), "rows") : src_rows;
    const int cols = as_extent(x.size(-1), "x") / (gate ? 2 : 1);
    const int32_t *at_rows = take ? (const int32_t *)take->data_ptr() : nullptr;
    Results out(call, a[5], form == BOTH ? 4 : 2);
    if (tiles) {
        const bool turned = form == TILES_T;
        const int64_t r = turned ? cols : rows, c = turned ? rows : cols;
        const std::vector<int64_t> shape = dims == 3 ? std::vector<int64_t>{count, r, c} : std::vector<int64_t>{r, c};
        const std::vector<int64_t> blocks = dims == 3 ? std::vector<int64_t>{count, blocks_of(r), blocks_of(c)} : std::vector<int64_t>{blocks_of(r), blocks_of(c)};
        const at::Tensor q = out.next(shape, at::kFloat8_e4m3fn, whole16(c), x, "values"), s = out.dense(blocks, at::kFloat, x, "scales");
        const int64_t ldq = row_distance(q, "values");
        if (dims == 3 && count > 1 && q.stride(0) != r * ldq) refuse(PyExc_ValueError, "the matrices of the values must follow one another");
        run("quantize_fp8_tiles", lib.quantize_fp8_tiles, as_extent(count, "x"), rows, cols, x.data_ptr(), type, ld, turned, (uint8_t *)q.data_ptr(), ldq, (float *)s.data_ptr(), call.handle());
        return out.result();
    }
    at::Tensor q;
    at::Tensor s;
    if (form != COLUMNS) {
        q = out.next({rows, cols}, at::kFloat8_e4m3fn, whole16(cols), x, "values");
        s = out.dense({blocks_of(cols), rows}, at::kFloat, x, "scales");
    }
    if (form == ROWS) {
        run("quantize_fp8_rows", lib.quantize_fp8_rows, rows, cols, x.data_ptr(), type, ld, gate, at_rows, per_row, src_rows, (uint8_t *)q.data_ptr(), row_distance(q, "values"),
            (float *)s.data_ptr(), call.handle());
        return out.result();
    }
    const at::Tensor qt = out.next({cols, rows}, at::kFloat8_e4m3fn, whole16(rows), x, "transposed values");
    const at::Tensor st = out.dense({blocks_of(rows), cols}, at::kFloat, x, "columns' scales");
    const bool both = form == BOTH;
    run("quantize_fp8_columns", lib.quantize_fp8_columns, rows, cols, x.data_ptr(), type, ld, gate, at_rows, per_row, src_rows, (uint8_t *)qt.data_ptr(),
        row_distance(qt, "transposed values"), (float *)st.data_ptr(), both ? (uint8_t *)q.data_ptr() : nullptr,
        both ? row_distance(q, "values") : 0, both ? (float *)s.data_ptr() : nullptr, call.handle());
    return out.result();
})

// (x, dh, out, stream)
NATIVE(silu_gate_backward, 4, {
    Call call(a[3]);
    const at::Tensor &x = call.rows(a[0], 2, "x"), &dh = call.rows(a[1], 2, "dh");
    const int type = type_of(x, "x");
    if (dh.scalar_type() != x.scalar_type()) refuse(PyExc_TypeError, "x and dh must have one type");
    if (x.size(0) != dh.size(0) || x.size(1) != 2 * dh.size(1)) refuse(PyExc_ValueError, "x must have dh's rows and twice its columns");
    const int rows = as_extent(x.size(0), "x"), cols = as_extent(dh.size(1), "dh");
    Results out(call, a[2], 1);
    const at::Tensor dx = out.next({rows, 2 * (int64_t)cols}, x.scalar_type(), 0, x, "out");
    run("silu_gate_backward", lib.silu_gate_backward, rows, cols, x.data_ptr(), row_distance(x, "x"), dh.data_ptr(), row_distance(dh, "dh"), dx.data_ptr(), row_distance(dx, "out"), type,
        call.handle());
    return out.result();
})

at::ScalarType as_dtype(PyObject *o)
{
    if (!THPDtype_Check(o)) refuse(PyExc_TypeError, "dtype must be a torch.dtype");
    const at::ScalarType t = reinterpret_cast<THPDtype *>(o)->scalar_type;
    if (type_of(t) < 0) refuse(PyExc_TypeError, "dtype must be float32, bfloat16 or float16");
    return t;
}

// (a, a_scale, b, b_scale, b_rows, dtype, fast_sums, out, stream)
NATIVE(gemm_fp8_nt, 9, {
    Call call(a[8]);
    const int fast_sums = as_bool(a[6]);
    const at::Tensor &A = call.e4m3(a[0], 2, "a"), &B = call.e4m3(a[2], 2, "b");
    if (A.size(1) != B.size(1)) refuse(PyExc_ValueError, "a and b must have one depth");
    const int M = as_extent(A.size(0), "a"), N = as_extent(B.size(0), "b"), K = as_extent(A.size(1), "a");
    const bool b_rows = as_bool(a[4]);
    const at::Tensor &sa = call.dense(a[1], at::kFloat, {blocks_of(K), M}, "a_scale");
    const at::Tensor &sb = b_rows ? call.dense(a[3], at::kFloat, {blocks_of(K), N}, "b_scale") : call.dense(a[3], at::kFloat, {blocks_of(N), blocks_of(K)}, "b_scale");
    const at::ScalarType dtype = as_dtype(a[5]);
    Results out(call, a[7], 1);
    const at::Tensor C = out.next({M, N}, dtype, 0, A, "out");
    run("gemm_fp8_nt", lib.gemm_fp8_nt, M, N, K, (const uint8_t *)A.data_ptr(), row_distance(A, "a"), (const float *)sa.data_ptr(), (const uint8_t *)B.data_ptr(),
        row_distance(B, "b"), (const float *)sb.data_ptr(), b_rows, C.data_ptr(), row_distance(C, "out"), type_of(dtype), fast_sums, call.handle());
    return out.result();
})

// (a, a_scale, w, w_scale, offsets, rows, per_row, dtype, fast_sums, out, stream)
NATIVE(gemm_fp8_experts, 11, {
    Call call(a[10]);
    const int fast_sums = as_bool(a[8]);
    const at::Tensor &A = call.e4m3(a[0], 2, "a"), &W = call.e4m3(a[2], 3, "w");
    if (A.size(1) != W.size(2)) refuse(PyExc_ValueError, "a and w must have one depth");
    const int a_rows = as_extent(A.size(0), "a"), E = as_extent(W.size(0), "w"), N = as_extent(W.size(1), "w"), K = as_extent(A.size(1), "a");
    const at::Tensor &sa = call.dense(a[1], at::kFloat, {blocks_of(K), a_rows}, "a_scale"),
                     &sw = call.dense(a[3], at::kFloat, {E, blocks_of(N), blocks_of(K)}, "w_scale"),
                     &offsets = call.dense(a[4], at::kInt, {E + 1}, "offsets");
    const int64_t ldw = row_distance(W, "w");
    if (E > 1 && W.stride(0) != N * ldw) refuse(PyExc_ValueError, "the matrices of w must follow one another");
    const at::Tensor *rows = nullptr;
    if (a[5] != Py_None) {
        rows = &call.on_device(tensor(a[5], "rows"), "rows");
        if (rows->scalar_type() != at::kInt || rows->dim() != 1 || !rows->is_contiguous()) refuse(PyExc_TypeError, "rows must be a contiguous int32 vector");
    }
    const int R = rows ? as_extent(rows->size(0), "rows") : a_rows, per_row = whole(a[6], "per_row");
    const at::ScalarType dtype = as_dtype(a[7]);
    Results out(call, a[9], 1);
    const at::Tensor C = out.next({R, N}, dtype, 0, A, "out");
    run("gemm_fp8_experts", lib.gemm_fp8_experts, R, a_rows, E, N, K, (const uint8_t *)A.data_ptr(), row_distance(A, "a"), (const float *)sa.data_ptr(), (const uint8_t *)W.data_ptr(),
        ldw, (const float *)sw.data_ptr(), (const int32_t *)offsets.data_ptr(), rows ? (const int32_t *)rows->data_ptr() : nullptr, per_row,
        C.data_ptr(), row_distance(C, "out"), type_of(dtype), fast_sums, call.handle());
    return out.result();
})

// (a, a_scale, b, b_scale, offsets, dtype, fast_sums, out, stream)
NATIVE(gemm_fp8_experts_grad, 9, {
    Call call(a[8]);
    const int fast_sums = as_bool(a[6]);
    const at::Tensor &A = call.e4m3(a[0], 2, "a"), &B = call.e4m3(a[2], 2, "b");
    if (A.size(1) != B.size(1)) refuse(PyExc_ValueError, "a and b must have one depth");
    const int N = as_extent(A.size(0), "a"), K = as_extent(B.size(0), "b"), R = as_extent(A.size(1), "a");
    const at::Tensor &sa = call.dense(a[1], at::kFloat, {blocks_of(R), N}, "a_scale"), &sb = call.dense(a[3], at::kFloat, {blocks_of(R), K}, "b_scale");
    const at::Tensor &off = call.on_device(tensor(a[4], "offsets"), "offsets");
    if (off.scalar_type() != at::kInt || off.dim() != 1 || off.size(0) < 2 || !off.is_contiguous())
        refuse(PyExc_TypeError, "offsets must be a contiguous int32 vector of one more than the experts");
    const int E = as_extent(off.size(0), "offsets") - 1;
    const at::ScalarType dtype = as_dtype(a[5]);
    Results out(call, a[7], 1);
    const at::Tensor C = out.next({E, N, K}, dtype, 0, A, "out");
    const int64_t ldc = row_distance(C, "out");
    if (E > 1 && C.stride(0) != N * ldc) refuse(PyExc_ValueError, "the matrices of out must follow one another");
    run("gemm_fp8_experts_grad", lib.gemm_fp8_experts_grad, R, E, N, K, (const uint8_t *)A.data_ptr(), row_distance(A, "a"), (const float *)sa.data_ptr(), (const uint8_t *)B.data_ptr(),
        row_distance(B, "b"), (const float *)sb.data_ptr(), (const int32_t *)off.data_ptr(), C.data_ptr(), ldc, type_of(dtype), fast_sums, call.handle());
    return out.result();
})

float as_float(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyFail{};
    return (float)v;
}

// (logits, k, sigmoid, bias, groups, kept, group_top, renormalise, factor, out, stream)
NATIVE(route_experts, 11, {
    Call call(a[10]);
    const at::Tensor &x = call.rows(a[0], 2, "logits");
    const int type = type_of(x, "logits"), T = as_extent(x.size(0), "logits"), E = as_extent(x.size(1), "logits"), k = whole(a[1], "k");
    const at::Tensor *bias = a[3] == Py_None ? nullptr : &call.dense(a[3], at::kFloat, {E}, "bias");
    const int sigmoid = as_bool(a[2]), groups = whole(a[4], "groups"), kept = whole(a[5], "kept"), group_top = whole(a[6], "group_top"), renormalise = as_bool(a[7]);
    const float factor = as_float(a[8]);
    if (k < 1 || k > EXPERTS_MOST_CHOICES) fail(CONV_ERR_INVALID_ARG, "route_experts");
    Results out(call, a[9], 2);
    const at::Tensor ids = out.dense({T, k}, at::kInt, x, "ids"), weights = out.dense({T, k}, at::kFloat, x, "weights");
    run("route_experts", lib.route_experts, T, E, k, x.data_ptr(), type, row_distance(x, "logits"), bias ? (const float *)bias->data_ptr() : nullptr, sigmoid, groups, kept, group_top,
        renormalise, factor, (int32_t *)ids.data_ptr(), (float *)weights.data_ptr(), call.handle());
    return out.result();
})

// (dweights, ids, logits, sigmoid, renormalise, factor, out, stream)
NATIVE(route_experts_backward, 8, {
    Call call(a[7]);
    const at::Tensor &x = call.rows(a[2], 2, "logits"), &ids = call.on_device(tensor(a[1], "ids"), "ids");
    require_dims(ids, 2, "ids");
    const int type = type_of(x, "logits"), T = as_extent(x.size(0), "logits"), E = as_extent(x.size(1), "logits"), k = as_extent(ids.size(1), "ids");
    call.dense(a[1], at::kInt, {T, k}, "ids");
    const at::Tensor &dw = call.dense(a[0], at::kFloat, {T, k}, "dweights");
    const int sigmoid = as_bool(a[3]), renormalise = as_bool(a[4]);
    const float factor = as_float(a[5]);
    Results out(call, a[6], 1);
    const at::Tensor dx = out.next({T, E}, x.scalar_type(), 0, x, "out");
    run("route_experts_backward", lib.route_experts_backward, T, E, k, x.data_ptr(), type, row_distance(x, "logits"), (const int32_t *)ids.data_ptr(), (const float *)dw.data_ptr(), sigmoid,
        renormalise, factor, dx.data_ptr(), row_distance(dx, "out"), call.handle());
    return out.result();
})

// (ids, experts, align, out, stream)
NATIVE(expert_rows, 5, {
    Call call(a[4]);
    const at::Tensor &ids = call.on_device(tensor(a[0], "ids"), "ids");
    if (ids.scalar_type() != at::kInt || !ids.is_contiguous()) refuse(PyExc_TypeError, "ids must be a contiguous int32 tensor");
    const int pairs = as_extent(ids.numel(), "ids"), E = whole(a[1], "experts"), align = whole(a[2], "align");
    const int R = lib.expert_rows_capacity(pairs, E, align);
    if (E < 1 || E > EXPERTS_MOST || (R == 0 && (pairs > 0 || align != 1))) fail(CONV_ERR_INVALID_ARG, "expert_rows");
    Results out(call, a[3], 3);
    const at::Tensor offsets = out.dense({E + 1}, at::kInt, ids, "offsets"), rows = out.dense({R}, at::kInt, ids, "rows"),
                     place = out.dense(ids.sizes(), at::kInt, ids, "place");
    run("expert_rows", lib.expert_rows, pairs, E, align, (const int32_t *)ids.data_ptr(), (int32_t *)offsets.data_ptr(), (int32_t *)rows.data_ptr(), (int32_t *)place.data_ptr(),
        call.handle());
    return out.result();
})

// (y, place, weights, out, stream)
NATIVE(combine_experts, 5, {
    Call call(a[4]);
    const at::Tensor &y = call.rows(a[0], 2, "y"), &place = call.on_device(tensor(a[1], "place"), "place");
    require_dims(place, 2, "place");
    const int type = type_of(y, "y"), T = as_extent(place.size(0), "place"), k = as_extent(place.size(1), "place");
    const int R = as_extent(y.size(0), "y"), N = as_extent(y.size(1), "y");
    call.dense(a[1], at::kInt, {T, k}, "place");
    const at::Tensor *w = a[2] == Py_None ? nullptr : &call.dense(a[2], at::kFloat, {T, k}, "weights");
    Results out(call, a[3], 1);
    const at::Tensor o = out.next({T, N}, y.scalar_type(), 0, y, "out");
    run("combine_experts", lib.combine_experts, T, k, N, R, y.data_ptr(), row_distance(y, "y"), type, (const int32_t *)place.data_ptr(), w ? (const float *)w->data_ptr() : nullptr,
        o.data_ptr(), row_distance(o, "out"), call.handle());
    return out.result();
})

// (dout, y, place, rows, weights, out, stream)
NATIVE(combine_experts_backward, 7, {
    Call call(a[6]);
    const at::Tensor &d = call.rows(a[0], 2, "dout"), &y = call.rows(a[1], 2, "y"), &place = call.on_device(tensor(a[2], "place"), "place");
    require_dims(place, 2, "place");
    const int type = type_of(y, "y"), T = as_extent(place.size(0), "place"), k = as_extent(place.size(1), "place");
    const int R = as_extent(y.size(0), "y"), N = as_extent(y.size(1), "y");
    if (d.scalar_type() != y.scalar_type()) refuse(PyExc_TypeError, "dout and y must have one type");
    if (d.size(0) != T || d.size(1) != N) refuse(PyExc_ValueError, "dout must have place's rows and y's columns");
    call.dense(a[2], at::kInt, {T, k}, "place");
    const at::Tensor &rows = call.dense(a[3], at::kInt, {R}, "rows");
    const at::Tensor *w = a[4] == Py_None ? nullptr : &call.dense(a[4], at::kFloat, {T, k}, "weights");
    Results out(call, a[5], 2);
    const at::Tensor dy = out.next({R, N}, y.scalar_type(), 0, y, "out[0]"), dw = out.dense({T, k}, at::kFloat, y, "out[1]");
    run("combine_experts_backward", lib.combine_experts_backward, T, k, N, R, d.data_ptr(), row_distance(d, "dout"), y.data_ptr(), row_distance(y, "y"), type, (const int32_t *)place.data_ptr(),
        (const int32_t *)rows.data_ptr(), w ? (const float *)w->data_ptr() : nullptr, dy.data_ptr(), row_distance(dy, "out[0]"),
        (float *)dw.data_ptr(), call.handle());
    return out.result();
})

}  // namespace

void experts_library(void *handle)
{
    missing = nullptr;
#define CALL(name) \
    if (!(lib.name = reinterpret_cast<decltype(&::name)>(dlsym(handle, #name)))) missing = #name;
    LIBRARY_CALLS(CALL)
#undef CALL
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr}
PyMethodDef experts_methods[] = {ENTRY(quantize_fp8), ENTRY(silu_gate_backward), ENTRY(gemm_fp8_nt), ENTRY(gemm_fp8_experts), ENTRY(gemm_fp8_experts_grad),
                                 ENTRY(route_experts), ENTRY(route_experts_backward), ENTRY(expert_rows), ENTRY(combine_experts), ENTRY(combine_experts_backward),
                                 {nullptr, nullptr, 0, nullptr}};
