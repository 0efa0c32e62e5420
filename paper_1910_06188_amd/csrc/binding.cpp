// Python entry points of the C ABI (include/q8.h): tensors to device pointers, numbers to the types of the declaration, the
// call with the interpreter lock released.  Sizes are checked by the Python functions in front, those of the 4-bit, grouped and routing
// entry points here.
//
// A call of a small layer is bound by the host: a kernel launch takes 3.5 us of it, and reading twelve tensors through three
// attribute calls each and handing eighteen arguments to ctypes took another 2.0 to 2.4.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>
#include <string>
#include <tuple>
#include <type_traits>
#include <utility>

#include "q8.h"

namespace {

// One argument.  On failure a Python error is set.
template <class T>
T argument(PyObject* o)
{
    if constexpr (std::is_pointer_v<T>) {
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "q8 takes tensors");
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        // of floats of two bytes and one the calls would read and write as many elements of four
        if (std::is_same_v<std::remove_cv_t<std::remove_pointer_t<T>>, float> && at::isFloatingType(t.scalar_type()) && t.element_size() < 4)
            PyErr_SetString(PyExc_TypeError, "q8 takes float32 tensors here");
        else if (!t.is_cuda())
            PyErr_SetString(PyExc_ValueError, "q8 takes device tensors");
        else if (!t.is_contiguous())
            PyErr_SetString(PyExc_ValueError, "q8 takes contiguous tensors");
        else
            return static_cast<T>(t.data_ptr());
        return nullptr;
    } else if constexpr (std::is_floating_point_v<T>) {
        return static_cast<T>(PyFloat_AsDouble(o));
    } else {
        return static_cast<T>(PyLong_AsUnsignedLongLongMask(o));
    }
}

// The stream, the last parameter of every function, comes as its raw handle; None is torch's current one.
void* stream_of(PyObject* o)
{
    if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
    return reinterpret_cast<void*>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLongMask(o)));
}

template <auto kFunction, class... A, size_t... I>
PyObject* call(PyObject* const* args, q8_status (*)(A...), std::index_sequence<I...>)
{
    using Params = std::tuple<A...>;
    Params p;
    constexpr size_t kStream = sizeof...(A) - 1;
    const auto convert = [&](auto index) {
        constexpr size_t i = decltype(index)::value;
        if constexpr (i == kStream)
            std::get<i>(p) = stream_of(args[i]);
        else
            std::get<i>(p) = argument<std::tuple_element_t<i, Params>>(args[i]);
        return PyErr_Occurred() == nullptr;
    };
    if (!(convert(std::integral_constant<size_t, I>{}) && ...)) return nullptr;
    q8_status status;
    Py_BEGIN_ALLOW_THREADS
    status = std::apply(kFunction, p);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(static_cast<long>(status));
}

template <class... A>
constexpr size_t arity(q8_status (*)(A...))
{
    return sizeof...(A);
}

template <auto kFunction>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    constexpr size_t kArgs = arity(kFunction);
    if (n != static_cast<Py_ssize_t>(kArgs)) return PyErr_Format(PyExc_TypeError, "takes %zu arguments, got %zd", kArgs, n);
    try {
        return call<kFunction>(args, kFunction, std::make_index_sequence<kArgs>{});
    } catch (const std::exception& e) {  // a tensor without storage of its own (under a functional transform)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// ---- entry points of tensors: shapes, element types and devices are looked at here, which in Python took as long as the launch ----

struct Refused {
    PyObject* type;
    std::string text;
};
[[noreturn]] void refuse(PyObject* type, const char* where, const std::string& what) { throw Refused{type, std::string(where) + ": " + what}; }

const at::Tensor& tensor(PyObject* o, const char* where)
{
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, where, "takes tensors");
    return THPVariable_Unpack(o);
}
const at::Tensor* tensor_or_none(PyObject* o, const char* where) { return o == Py_None ? nullptr : &tensor(o, where); }

// The address of a tensor of type `type` on the current device, the one that the call's stream and kernels are on.
void* address(const at::Tensor& t, at::ScalarType type, const char* where)
{
    if (t.scalar_type() != type) refuse(PyExc_TypeError, where, std::string("takes a tensor of ") + at::toString(type) + " here, not " + at::toString(t.scalar_type()));
    if (!t.is_cuda()) refuse(PyExc_ValueError, where, "takes device tensors");
    if (!t.is_contiguous()) refuse(PyExc_ValueError, where, "takes contiguous tensors");
    if (t.get_device() != c10::hip::current_device()) refuse(PyExc_ValueError, where, "takes tensors of the current device");
    return t.data_ptr();
}
template <class T>
T* data(const at::Tensor& t, const char* where)
{
    if constexpr (std::is_same_v<T, float>)
        return static_cast<T*>(address(t, at::kFloat, where));
    else if constexpr (std::is_same_v<T, int8_t>)
        return static_cast<T*>(address(t, at::kChar, where));
    else if constexpr (std::is_same_v<T, uint8_t>)
        return static_cast<T*>(address(t, at::kByte, where));
    else
        return static_cast<T*>(address(t, at::kInt, where));
}
template <class T>
T* data(const at::Tensor* t, const char* where)
{
    return t ? data<T>(*t, where) : nullptr;
}

int float_type(const at::Tensor& t, const char* where)
{
    if (t.scalar_type() == at::kFloat) return Q8_TYPE_F32;
    if (t.scalar_type() == at::kBFloat16) return Q8_TYPE_BF16;
    refuse(PyExc_TypeError, where, std::string("takes float32 or bfloat16, not ") + at::toString(t.scalar_type()));
}
void* float_data(const at::Tensor& t, const char* where) { return address(t, t.scalar_type(), where); }

struct Pending {};  // a Python error is set

uint32_t flags_of(PyObject* o)
{
    const uint32_t flags = static_cast<uint32_t>(PyLong_AsUnsignedLongMask(o));
    if (PyErr_Occurred()) throw Pending{};
    return flags;
}

// Codes [.., rows, 64 G] and scales [.., G, rows, 4], `dims` dimensions of codes.
void check_mx4(const at::Tensor& codes, const at::Tensor& scales, int64_t dims, const char* where)
{
    bool fit = codes.dim() == dims && scales.dim() == dims + 1;
    if (fit) {
        const auto c = codes.sizes(), s = scales.sizes();
        fit = c[dims - 1] % 64 == 0 && s[dims - 2] == c[dims - 1] / 64 && s[dims - 1] == c[dims - 2] && s[dims] == 4 && (dims == 2 || s[0] == c[0]);
    }
    if (!fit) refuse(PyExc_ValueError, where, "codes [.., rows, 64 G] and scales [.., G, rows, 4] do not fit each other");
}

// The output of a 4-bit product: codes if there are scales for them, else fp32 or bf16.
int product_output(const at::Tensor& y, const at::Tensor* y_scales, int64_t M, int64_t N, const char* where)
{
    if (!y_scales) {
        if (y.dim() != 2 || y.size(0) != M || y.size(1) != N) refuse(PyExc_ValueError, where, "y is [rows, N]");
        return float_type(y, where);
    }
    if (y.scalar_type() != at::kByte) refuse(PyExc_TypeError, where, "codes are uint8");
    if (N % 128 != 0 || y.dim() != 2 || y.size(0) != M || y.size(1) != N / 2) refuse(PyExc_ValueError, where, "4-bit outputs are codes [rows, N / 2] of a width that is a multiple of 128");
    check_mx4(y, *y_scales, 2, where);
    return Q8_TYPE_MX4;
}

template <class F>
q8_status unlocked(F&& f)
{
    q8_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f();
    Py_END_ALLOW_THREADS
    return s;
}

struct mx4_quantize {  // x, codes, scales, stream
    static constexpr int kArgs = 4;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &x = tensor(a[0], where), &codes = tensor(a[1], where), &scales = tensor(a[2], where);
        if (x.dim() != 2) refuse(PyExc_ValueError, where, "x is [rows, K]");
        const int64_t M = x.size(0), K = x.size(1);
        check_mx4(codes, scales, 2, where);
        if (codes.size(0) != M || codes.size(1) != Q8_MX4_CODE_BYTES(K)) refuse(PyExc_ValueError, where, "codes and scales do not fit x");
        const int type = float_type(x, where);
        void* xp = float_data(x, where);
        uint8_t *c = data<uint8_t>(codes, where), *s = data<uint8_t>(scales, where);
        void* st = stream_of(a[3]);
        return unlocked([&] { return q8_mx4_quantize(xp, type, M, K, c, s, st); });
    }
};
struct mx4_fake_quantize {  // x, xq, stream
    static constexpr int kArgs = 3;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &x = tensor(a[0], where), &xq = tensor(a[1], where);
        if (x.dim() != 2 || xq.sizes() != x.sizes() || xq.scalar_type() != x.scalar_type()) refuse(PyExc_ValueError, where, "xq and x are [rows, K] of one type");
        const int64_t M = x.size(0), K = x.size(1);
        const int type = float_type(x, where);
        void *xp = float_data(x, where), *q = float_data(xq, where), *st = stream_of(a[2]);
        return unlocked([&] { return q8_mx4_fake_quantize(xp, type, M, K, q, st); });
    }
};
struct mx4_ste_backward {  // grad_xq, grad_x, stream
    static constexpr int kArgs = 3;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &g = tensor(a[0], where), &gx = tensor(a[1], where);
        if (gx.scalar_type() != g.scalar_type()) refuse(PyExc_TypeError, where, "the gradients are of one type");
        if (gx.numel() != g.numel()) refuse(PyExc_ValueError, where, "sizes differ");
        const int64_t n = g.numel();
        const int type = float_type(g, where);
        void *from = float_data(g, where), *to = float_data(gx, where), *st = stream_of(a[2]);
        return unlocked([&] { return q8_mx4_ste_backward(from, type, n, to, st); });
    }
};
struct mx4_linear {  // xq, xs, wq, ws, bias, y, y_scales, flags, stream
    static constexpr int kArgs = 9;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &xq = tensor(a[0], where), &xs = tensor(a[1], where), &wq = tensor(a[2], where), &ws = tensor(a[3], where), &y = tensor(a[5], where);
        const at::Tensor *bias = tensor_or_none(a[4], where), *y_scales = tensor_or_none(a[6], where);
        check_mx4(xq, xs, 2, where);
        check_mx4(wq, ws, 2, where);
        const int64_t M = xq.size(0), N = wq.size(0), K = 2 * xq.size(1);
        if (wq.size(1) != xq.size(1) || (bias && bias->numel() != N)) refuse(PyExc_ValueError, where, "x, w and bias do not fit each other");
        const int type = product_output(y, y_scales, M, N, where);
        const uint8_t *c = data<uint8_t>(xq, where), *s = data<uint8_t>(xs, where), *w = data<uint8_t>(wq, where), *v = data<uint8_t>(ws, where);
        const float* b = data<float>(bias, where);
        void *yp = float_data(y, where), *st = stream_of(a[8]);
        uint8_t* ys = data<uint8_t>(y_scales, where);
        const uint32_t flags = flags_of(a[7]);
        return unlocked([&] { return q8_mx4_linear(c, s, w, v, b, M, N, K, yp, type, ys, flags, st); });
    }
};
struct mx4_linear_dynamic {  // x, wq, ws, bias, xq_work, xs_work, y, y_scales, flags, stream
    static constexpr int kArgs = 10;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &x = tensor(a[0], where), &wq = tensor(a[1], where), &ws = tensor(a[2], where), &cw = tensor(a[4], where), &sw = tensor(a[5], where), &y = tensor(a[6], where);
        const at::Tensor *bias = tensor_or_none(a[3], where), *y_scales = tensor_or_none(a[7], where);
        if (x.dim() != 2) refuse(PyExc_ValueError, where, "x is [rows, K]");
        check_mx4(wq, ws, 2, where);
        const int64_t M = x.size(0), K = x.size(1), N = wq.size(0);
        if (wq.size(1) != Q8_MX4_CODE_BYTES(K) || (bias && bias->numel() != N)) refuse(PyExc_ValueError, where, "x, w and bias do not fit each other");
        if (cw.numel() < M * Q8_MX4_CODE_BYTES(K) || sw.numel() < M * Q8_MX4_SCALE_BYTES(K)) refuse(PyExc_ValueError, where, "scratch of mx4_empty(M, K) needed");
        const int x_type = float_type(x, where), type = product_output(y, y_scales, M, N, where);
        const void* xp = float_data(x, where);
        const uint8_t *w = data<uint8_t>(wq, where), *v = data<uint8_t>(ws, where);
        const float* b = data<float>(bias, where);
        uint8_t *c = data<uint8_t>(cw, where), *s = data<uint8_t>(sw, where), *ys = data<uint8_t>(y_scales, where);
        void *yp = float_data(y, where), *st = stream_of(a[9]);
        const uint32_t flags = flags_of(a[8]);
        return unlocked([&] { return q8_mx4_linear_dynamic(xp, x_type, w, v, b, M, N, K, c, s, yp, type, ys, flags, st); });
    }
};

// The arguments that the grouped products share: rows of x, and which of them the M rows of y read.
void check_rows(const at::Tensor& x, const at::Tensor* x_rows, int64_t M, const char* where)
{
    if ((x_rows ? x_rows->numel() : x.size(0)) != M) refuse(PyExc_ValueError, where, "x_rows, or x without it, has as many rows as y");
}
struct mx4_linear_grouped {  // xq, xs, wq, ws, bias, group_rows, y, x_rows, y_scales, flags, stream
    static constexpr int kArgs = 11;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &xq = tensor(a[0], where), &xs = tensor(a[1], where), &wq = tensor(a[2], where), &ws = tensor(a[3], where), &rows = tensor(a[5], where), &y = tensor(a[6], where);
        const at::Tensor *bias = tensor_or_none(a[4], where), *x_rows = tensor_or_none(a[7], where), *y_scales = tensor_or_none(a[8], where);
        check_mx4(xq, xs, 2, where);
        check_mx4(wq, ws, 3, where);
        if (y.dim() != 2) refuse(PyExc_ValueError, where, "y is [rows, N]");
        const int64_t n = xq.size(0), E = wq.size(0), N = wq.size(1), K = 2 * xq.size(1), M = y.size(0);
        if (wq.size(2) != xq.size(1) || rows.numel() != E || (bias && bias->numel() != E * N)) refuse(PyExc_ValueError, where, "x, w, bias and group_rows do not fit each other");
        check_rows(xq, x_rows, M, where);
        const int type = product_output(y, y_scales, M, N, where);
        const uint8_t *c = data<uint8_t>(xq, where), *s = data<uint8_t>(xs, where), *w = data<uint8_t>(wq, where), *v = data<uint8_t>(ws, where);
        const float* b = data<float>(bias, where);
        const int32_t *g = data<int32_t>(rows, where), *r = data<int32_t>(x_rows, where);
        void *yp = float_data(y, where), *st = stream_of(a[10]);
        uint8_t* ys = data<uint8_t>(y_scales, where);
        const uint32_t flags = flags_of(a[9]);
        return unlocked([&] { return q8_mx4_linear_grouped(c, s, n, r, w, v, b, g, (int)std::min<int64_t>(E, INT_MAX), M, N, K, yp, type, ys, flags, st); });
    }
};
struct linear_grouped {  // xq, wq, bias, sx, sw, group_rows, y, x_rows, out_amax, next_scale, flags, stream
    static constexpr int kArgs = 12;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &xq = tensor(a[0], where), &wq = tensor(a[1], where), &sx = tensor(a[3], where), &sw = tensor(a[4], where), &rows = tensor(a[5], where), &y = tensor(a[6], where);
        const at::Tensor *bias = tensor_or_none(a[2], where), *x_rows = tensor_or_none(a[7], where), *amax = tensor_or_none(a[8], where), *next = tensor_or_none(a[9], where);
        const uint32_t flags = flags_of(a[10]);
        if (xq.dim() != 2 || wq.dim() != 3 || y.dim() != 2) refuse(PyExc_ValueError, where, "x is [rows, K], w [experts, N, K], y [rows, N]");
        const int64_t n = xq.size(0), K = xq.size(1), E = wq.size(0), N = wq.size(1), M = y.size(0);
        if (wq.size(2) != K || y.size(1) != N || rows.numel() != E || sx.numel() < 1 || sw.numel() != E || (bias && bias->numel() != E * N) || (amax && amax->numel() < 1) || (next && next->numel() < 1))
            refuse(PyExc_ValueError, where, "x, w, bias, scales, group_rows and y do not fit each other");
        check_rows(xq, x_rows, M, where);
        const at::ScalarType type = flags & Q8_EPI_REQUANT ? at::kChar : at::kFloat;
        if (y.scalar_type() != type) refuse(PyExc_ValueError, where, "y is float32, or int8 with EPI_REQUANT");
        const int8_t *x = data<int8_t>(xq, where), *w = data<int8_t>(wq, where);
        const float *b = data<float>(bias, where), *s = data<float>(sx, where), *v = data<float>(sw, where), *ns = data<float>(next, where);
        const int32_t *g = data<int32_t>(rows, where), *r = data<int32_t>(x_rows, where);
        float* am = data<float>(amax, where);
        void *yp = address(y, type, where), *st = stream_of(a[11]);
        return unlocked([&] { return q8_linear_grouped(x, n, r, w, b, s, v, g, (int)std::min<int64_t>(E, INT_MAX), M, N, K, yp, am, ns, flags, st); });
    }
};
struct route {  // logits, experts, gates, group_rows, rows, slots, work, stream
    static constexpr int kArgs = 8;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &logits = tensor(a[0], where), &experts = tensor(a[1], where), &gates = tensor(a[2], where), &counts = tensor(a[3], where), &rows = tensor(a[4], where),
                         &slots = tensor(a[5], where), &work = tensor(a[6], where);
        if (logits.dim() != 2 || experts.dim() != 2) refuse(PyExc_ValueError, where, "logits are [tokens, experts], experts [tokens, k]");
        const int64_t T = logits.size(0), E = logits.size(1), k = experts.size(1);
        if (experts.size(0) != T || gates.numel() != T * k || counts.numel() != E || rows.numel() != T * k || slots.numel() != T * k) refuse(PyExc_ValueError, where, "the outputs do not fit the logits");
        if (work.numel() < Q8_ROUTE_BLOCKS * E) refuse(PyExc_ValueError, where, "work holds ROUTE_BLOCKS * n_experts integers");
        const float* l = data<float>(logits, where);
        float* g = data<float>(gates, where);
        int32_t *e = data<int32_t>(experts, where), *c = data<int32_t>(counts, where), *r = data<int32_t>(rows, where), *s = data<int32_t>(slots, where), *w = data<int32_t>(work, where);
        void* st = stream_of(a[7]);
        return unlocked([&] { return q8_route(l, T, (int)std::min<int64_t>(E, INT_MAX), (int)std::min<int64_t>(k, INT_MAX), e, g, c, r, s, w, st); });
    }
};
struct combine {  // y, slots, gates, out, stream
    static constexpr int kArgs = 5;
    static q8_status run(PyObject* const* a, const char* where)
    {
        const at::Tensor &y = tensor(a[0], where), &slots = tensor(a[1], where), &gates = tensor(a[2], where), &out = tensor(a[3], where);
        if (y.dim() != 2 || slots.dim() != 2 || out.dim() != 2 || gates.numel() != slots.numel() || out.size(0) != slots.size(0) || out.size(1) != y.size(1) || out.scalar_type() != y.scalar_type())
            refuse(PyExc_ValueError, where, "y is [rows, N], slots and gates [tokens, k], out [tokens, N] of y's type");
        const int64_t R = y.size(0), T = slots.size(0), k = slots.size(1), N = y.size(1);
        const int type = float_type(y, where);
        const void* yp = float_data(y, where);
        const int32_t* s = data<int32_t>(slots, where);
        const float* g = data<float>(gates, where);
        void *o = float_data(out, where), *st = stream_of(a[4]);
        return unlocked([&] { return q8_combine(yp, R, s, g, T, (int)std::min<int64_t>(k, INT_MAX), N, o, type, st); });
    }
};

template <class Entry>
struct Name;
#define Q8_NAME(NAME) \
    template <>       \
    struct Name<NAME> { static constexpr const char* kText = "q8_" #NAME; }
Q8_NAME(mx4_quantize);
Q8_NAME(mx4_fake_quantize);
Q8_NAME(mx4_ste_backward);
Q8_NAME(mx4_linear);
Q8_NAME(mx4_linear_dynamic);
Q8_NAME(mx4_linear_grouped);
Q8_NAME(linear_grouped);
Q8_NAME(route);
Q8_NAME(combine);
#undef Q8_NAME

template <class Entry>
PyObject* checked(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != Entry::kArgs) return PyErr_Format(PyExc_TypeError, "takes %d arguments, got %zd", Entry::kArgs, n);
    if (args[n - 1] != Py_None) {  // no launch on what is no handle
        stream_of(args[n - 1]);
        if (PyErr_Occurred()) return nullptr;
    }
    try {
        return PyLong_FromLong(static_cast<long>(Entry::run(args, Name<Entry>::kText)));
    } catch (const Pending&) {
    } catch (const Refused& r) {
        PyErr_SetString(r.type, r.text.c_str());
    } catch (const std::exception& e) {  // a tensor without storage of its own (under a functional transform)
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

#define Q8_ENTRY(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<&NAME>)), METH_FASTCALL, nullptr}
#define Q8_CHECKED_ENTRY(NAME) {"q8_" #NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&checked<NAME>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {Q8_ENTRY(q8_absmax),
                         Q8_ENTRY(q8_scale_from_amax),
                         Q8_ENTRY(q8_quantize),
                         Q8_ENTRY(q8_quantize_amax),
                         Q8_ENTRY(q8_quantize_dynamic),
                         Q8_ENTRY(q8_linear),
                         Q8_ENTRY(q8_linear_residual),
                         Q8_ENTRY(q8_linear_f32),
                         Q8_ENTRY(q8_linear_f32_static),
                         Q8_ENTRY(q8_linear_f32_slots),
                         Q8_ENTRY(q8_embedding),
                         Q8_ENTRY(q8_embedding_sum3),
                         Q8_ENTRY(q8_fake_quantize),
                         Q8_ENTRY(q8_ema_update),
                         Q8_ENTRY(q8_fake_quantize_ema),
                         Q8_ENTRY(q8_ste_backward),
                         Q8_ENTRY(q8_layernorm_absmax),
                         Q8_ENTRY(q8_embedding_sum3_layernorm),
                         Q8_ENTRY(q8_attention),
                         Q8_CHECKED_ENTRY(mx4_quantize),
                         Q8_CHECKED_ENTRY(mx4_fake_quantize),
                         Q8_CHECKED_ENTRY(mx4_ste_backward),
                         Q8_CHECKED_ENTRY(mx4_linear),
                         Q8_CHECKED_ENTRY(mx4_linear_dynamic),
                         Q8_CHECKED_ENTRY(mx4_linear_grouped),
                         Q8_CHECKED_ENTRY(linear_grouped),
                         Q8_CHECKED_ENTRY(route),
                         Q8_CHECKED_ENTRY(combine),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
