// The calls a model makes for every layer - quantize, linear, both in one - from Python objects to the C ABI without
// ctypes: checks, allocations and pointers in native code.  Small calls are bound by the host: through ctypes
// linear_fp16 of one token took 9.6 us, linear (two calls) 16.1, of which the launches are 3.2 each; here 5.7 and 10.2.  77
// tokens through a layer of K = 1920, N = 3003 by two calls 16.4 -> 10.9 us, a token through the 8B block 36.5 -> 34.3, where
// its kernels (31.5 us) are the bound.  The library's functions come in as addresses, so that whichever build of it the
// package has loaded is the one that runs.  Nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "mixllm.h"

namespace {

namespace py = pybind11;

decltype(&mixllm_query_sizes) query_sizes;
decltype(&mixllm_quantize_activations) quantize_activations;
decltype(&mixllm_mixed_linear_path) mixed_linear_path;
decltype(&mixllm_mixed_linear_fp16) mixed_linear_fp16;
decltype(&mixllm_mixed_linear_epilogue) mixed_linear_epilogue;
decltype(&mixllm_mixed_linear_fp16_epilogue) mixed_linear_fp16_epilogue;
decltype(&mixllm_route_workspace) route_workspace;
decltype(&mixllm_route_experts) route_experts;
decltype(&mixllm_experts_workspace) experts_workspace;
decltype(&mixllm_experts_linear) experts_linear;
decltype(&mixllm_experts_linear_fp16) experts_linear_fp16;
decltype(&mixllm_experts_combine) experts_combine;
decltype(&mixllm_experts_table_bytes) experts_table_bytes;

struct Refused {   // what an assertion of the Python side would say
    const char *what;
};

// the tensor behind an argument, or an undefined one for None
at::Tensor tensor(PyObject *o)
{
    if (o == Py_None) return at::Tensor();
    TORCH_CHECK_TYPE(THPVariable_Check(o), "expected a tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

// device address of a tensor's data; null for none and for an empty one
void *address(const at::Tensor &t)
{
    if (!t.defined() || t.numel() == 0) return nullptr;
    if (!t.is_cuda() || !t.is_contiguous()) throw Refused{"device, contiguous tensors only"};
    return t.data_ptr();
}

int32_t index(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return (int32_t)v;
}

// a descriptor's field: whatever int() makes a number of
int32_t number(PyObject *o)
{
    if (PyLong_CheckExact(o)) return index(o);
    const py::object i = py::reinterpret_steal<py::object>(PyNumber_Long(o));
    if (!i) throw python_error();
    return index(i.ptr());
}

// K, N, n8, w8_group, w8, w4, s8, s4, z4, perm of a packed layer, as they stand in the arguments
struct Layer {
    int32_t K, N, n8, w8_group;
    at::Tensor w8, w4, s8, s4, z4, perm;
    explicit Layer(PyObject *const *a)
        : K(number(a[0])), N(number(a[1])), n8(number(a[2])), w8_group(number(a[3])), w8(tensor(a[4])), w4(tensor(a[5])), s8(tensor(a[6])),
          s4(tensor(a[7])), z4(tensor(a[8])), perm(tensor(a[9]))
    {
    }
};

void half_matrix(const at::Tensor &x)
{
    if (!x.defined() || x.scalar_type() != at::kHalf || x.dim() != 2) throw Refused{"x: an fp16 matrix"};
}

// A buffer of the caller's holds `n` values of `type`, or the same number of integers of that width (raw bits): what the
// kernels read and write goes by the sizes of the call alone.  A missing buffer is left to the library.
void holds(const at::Tensor &t, at::ScalarType type, int64_t n, const char *what)
{
    if (!t.defined()) return;
    const bool bits = at::isIntegralType(t.scalar_type(), /*includeBool=*/true) && t.itemsize() == (int64_t)at::elementSize(type);
    if ((t.scalar_type() != type && !bits) || t.numel() < n) throw Refused{what};
}

// A subclass of Tensor, or a mode, may have a new_empty of its own: results are then allocated by it, so that they are of
// the type they would have in Python.
bool overrides_new_empty(PyObject *o)
{
    return !THPVariable_CheckExact(o) || at::impl::torch_function_mode_enabled();
}
at::Tensor new_empty_in_python(PyObject *o, const py::tuple &sizes, at::ScalarType type)
{
    const auto dtype = py::reinterpret_borrow<py::object>((PyObject *)torch::getTHPDtype(type));
    return tensor(py::handle(o).attr("new_empty")(sizes, py::arg("dtype") = dtype).ptr());
}
at::Tensor new_empty_in_python(PyObject *o, int64_t rows, int64_t columns, at::ScalarType type)
{
    return new_empty_in_python(o, py::make_tuple(rows, columns), type);
}

// f() with its C++ exceptions as Python ones.  The calls below release the interpreter while they allocate and launch; a
// status other than MIXLLM_OK comes back as a number.
template <typename F>
PyObject *run(Py_ssize_t n, Py_ssize_t expected, F &&f)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == expected, "expected ", expected, " arguments, got ", n);
    try {
        return f();
    } catch (const Refused &r) {
        PyErr_SetString(PyExc_AssertionError, r.what);
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// (A workspace's element count stands for its bytes: exact for the uint8 tensor it is meant to be, short of them, never
// beyond, for any other.)

// linear_fp16(x, <layer>, act_group, out, workspace, stream) -> y, or a status
PyObject *py_linear_fp16(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 15, [&]() -> PyObject * {
        const at::Tensor x = tensor(a[0]);
        const Layer L(a + 1);
        const int32_t act_group = number(a[11]);
        at::Tensor y = tensor(a[12]), ws = tensor(a[13]);
        void *stream = PyLong_AsVoidPtr(a[14]);
        half_matrix(x);
        holds(y, at::kHalf, x.size(0) * L.N, "y: an fp16 buffer of tokens x outputs");
        if (x.size(1) != L.K) throw Refused{"x has as many columns as the layer has inputs"};
        if (!y.defined() && overrides_new_empty(a[0])) y = new_empty_in_python(a[0], x.size(0), L.N, at::kHalf);
        int rc;
        {
            py::gil_scoped_release no_gil;
            const mixllm_desc d{(int32_t)x.size(0), L.K, L.N, L.n8, MIXLLM_GROUP, act_group, L.w8_group};
            if (!y.defined()) y = x.new_empty({x.size(0), L.N});
            rc = MIXLLM_OK;
            if (!ws.defined()) {
                mixllm_sizes s;
                rc = query_sizes(&d, &s);
                if (rc == MIXLLM_OK) ws = x.new_empty({(int64_t)s.workspace_bytes}, x.options().dtype(at::kByte));
            }
            if (rc == MIXLLM_OK)
                rc = mixed_linear_fp16(&d, address(x), address(L.w4), address(L.w8), address(L.s4), address(L.s8), address(L.z4),
                                       (const int32_t *)address(L.perm), address(y), address(ws), (size_t)ws.numel(), stream);
        }
        return rc == MIXLLM_OK ? THPVariable_Wrap(std::move(y)) : PyLong_FromLong(rc);
    });
}

// quantize_activations(x, act_group or None, (xq, xs) or None, stream) -> (xq, xs), or a status.  Only where no buffers are
// given at all are they allocated: one that is missing from a pair is refused by the library.
PyObject *py_quantize_activations(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 4, [&]() -> PyObject * {
        const at::Tensor x = tensor(a[0]);
        const bool per_token = a[1] == Py_None, allocate = a[2] == Py_None;
        int32_t act_group = per_token ? 0 : allocate ? index(a[1]) : number(a[1]);   // (a tensor's size is an integer)
        at::Tensor xq, xs;
        if (!allocate) {
            const py::object out = py::reinterpret_steal<py::object>(PySequence_Tuple(a[2]));
            if (!out) throw python_error();
            TORCH_CHECK_VALUE(PyTuple_GET_SIZE(out.ptr()) == 2, "out: two buffers, got ", PyTuple_GET_SIZE(out.ptr()));
            xq = tensor(PyTuple_GET_ITEM(out.ptr(), 0));
            xs = tensor(PyTuple_GET_ITEM(out.ptr(), 1));
        }
        void *stream = PyLong_AsVoidPtr(a[3]);
        half_matrix(x);
        const int32_t M = (int32_t)x.size(0), K = (int32_t)x.size(1);
        if (per_token) act_group = K;
        holds(xq, at::kChar, (int64_t)M * K, "xq: an int8 buffer of tokens x inputs");
        if (act_group > 0) holds(xs, at::kHalf, (int64_t)M * (K / act_group), "xs: an fp16 buffer of tokens x groups");
        if (allocate && act_group <= 0) throw Refused{"act_group is positive"};
        if (allocate && overrides_new_empty(a[0])) {
            xq = new_empty_in_python(a[0], M, K, at::kChar);
            xs = new_empty_in_python(a[0], M, K / act_group, at::kHalf);
        }
        int rc;
        {
            py::gil_scoped_release no_gil;
            if (allocate && !xq.defined()) {
                xq = x.new_empty({M, K}, x.options().dtype(at::kChar));
                xs = x.new_empty({M, K / act_group});
            }
            const mixllm_desc d{M, K, 1, 0, MIXLLM_GROUP, act_group, K};
            rc = quantize_activations(&d, address(x), (int8_t *)address(xq), address(xs), stream);
        }
        if (rc != MIXLLM_OK) return PyLong_FromLong(rc);
        PyObject *q = THPVariable_Wrap(std::move(xq));
        PyObject *s = q ? THPVariable_Wrap(std::move(xs)) : nullptr;
        PyObject *both = s ? PyTuple_Pack(2, q, s) : nullptr;
        Py_XDECREF(q);
        Py_XDECREF(s);
        return both;
    });
}

// mixed_linear(xq, xs, <layer>, path, out, workspace, stream) -> y, or a status
PyObject *py_mixed_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 16, [&]() -> PyObject * {
        const at::Tensor xq = tensor(a[0]), xs = tensor(a[1]);
        const Layer L(a + 2);
        const int32_t path = index(a[12]);
        at::Tensor y = tensor(a[13]);
        const at::Tensor ws = tensor(a[14]);
        void *stream = PyLong_AsVoidPtr(a[15]);
        if (!xq.defined() || xq.dim() != 2) throw Refused{"xq: a matrix"};
        const int64_t M = xq.size(0), K = xq.size(1);
        if (K != L.K || xs.size(0) != M) throw Refused{"xq, xs and the layer agree in their sizes"};
        if (xs.size(1) == 0) throw Refused{"xs has a column"};
        const int32_t act_group = (int32_t)(K / xs.size(1));
        holds(xq, at::kChar, M * K, "xq: an int8 matrix");
        if (act_group == K || act_group == MIXLLM_GROUP) {
            // as many scales as the library reads: 129 columns for 130 groups also divide to groups of 128
            holds(xs, at::kHalf, M * (K / act_group), "xs: fp16 scales, tokens x groups");
            if (xs.numel() != M * (K / act_group)) throw Refused{"xs: one scale per token and group"};
        }
        holds(y, at::kHalf, M * L.N, "y: an fp16 buffer of tokens x outputs");
        if (!y.defined() && overrides_new_empty(a[0])) y = new_empty_in_python(a[0], M, L.N, at::kHalf);
        int rc;
        {
            py::gil_scoped_release no_gil;
            if (!y.defined()) y = xq.new_empty({M, L.N}, xq.options().dtype(at::kHalf));
            const mixllm_desc d{(int32_t)M, L.K, L.N, L.n8, MIXLLM_GROUP, act_group, L.w8_group};
            rc = mixed_linear_path(&d, (const int8_t *)address(xq), address(xs), address(L.w4), address(L.w8), address(L.s4), address(L.s8),
                                   address(L.z4), (const int32_t *)address(L.perm), address(y), address(ws),
                                   ws.defined() ? (size_t)ws.numel() : 0, path, stream);
        }
        return rc == MIXLLM_OK ? THPVariable_Wrap(std::move(y)) : PyLong_FromLong(rc);
    });
}

// ---- the operators next to the linear: every tensor of a call lies on the current device, whose stream is passed ----

// the device of a call: that of its first operand, which has to be the current one
at::Device current(const at::Tensor &t, const char *what)
{
    if (!t.defined() || !t.is_cuda()) throw Refused{what};
    if (c10::impl::VirtualGuardImpl(t.device().type()).getDevice() != t.device()) throw Refused{"tensors of the current device"};
    return t.device();
}
// address of a tensor on that device; null for none and for an empty one
void *address(const at::Tensor &t, at::Device d)
{
    if (t.defined() && t.device() != d) throw Refused{"tensors of one device"};
    return address(t);
}
// an operand that is absent, or of this type and these sizes
void shaped(const at::Tensor &t, at::ScalarType type, std::initializer_list<int64_t> sizes, const char *what)
{
    if (t.defined() && (t.scalar_type() != type || t.sizes() != at::IntArrayRef(sizes))) throw Refused{what};
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

// bias, residual, activation, gated as they stand in the arguments, for `rows` outputs of a layer (or `layers` of them) of N
struct Epilogue {
    at::Tensor bias, residual;
    int32_t activation, gated;
    int64_t columns;   // of the output
    Epilogue(PyObject *const *a, int64_t rows, int64_t N, int64_t layers)
        : bias(tensor(a[0])), residual(tensor(a[1])), activation(number(a[2])), gated(truth(a[3])), columns(gated ? N / 2 : N)
    {
        if (layers) shaped(bias, at::kHalf, {layers, N}, "bias: fp16, experts x outputs");
        else shaped(bias, at::kHalf, {N}, "bias: fp16, one per output");
        shaped(residual, at::kHalf, {rows, columns}, "residual: fp16, of the result's shape");
    }
    mixllm_epilogue of(at::Device d) const { return mixllm_epilogue{address(bias, d), address(residual, d), activation, gated}; }
};

// linear_fp16_epilogue(x, <layer>, act_group, bias, residual, activation, gated, out, workspace, stream) -> y, or a status
PyObject *py_linear_fp16_epilogue(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 19, [&]() -> PyObject * {
        const at::Tensor x = tensor(a[0]);
        const Layer L(a + 1);
        const int32_t act_group = number(a[11]);
        half_matrix(x);
        const int64_t M = x.size(0);
        const Epilogue e(a + 12, M, L.N, 0);
        at::Tensor y = tensor(a[16]), ws = tensor(a[17]);
        void *stream = PyLong_AsVoidPtr(a[18]);
        const at::Device dev = current(x, "x: an fp16 matrix on the device");
        shaped(y, at::kHalf, {M, e.columns}, "out: fp16, tokens x outputs");
        if (x.size(1) != L.K) throw Refused{"x has as many columns as the layer has inputs"};
        if (!y.defined() && overrides_new_empty(a[0])) y = new_empty_in_python(a[0], M, e.columns, at::kHalf);
        int rc;
        {
            py::gil_scoped_release no_gil;
            const mixllm_desc d{(int32_t)M, L.K, L.N, L.n8, MIXLLM_GROUP, act_group, L.w8_group};
            if (!y.defined()) y = x.new_empty({M, e.columns});
            rc = MIXLLM_OK;
            if (!ws.defined()) {
                mixllm_sizes s;
                rc = query_sizes(&d, &s);
                if (rc == MIXLLM_OK) ws = x.new_empty({(int64_t)s.workspace_bytes}, x.options().dtype(at::kByte));
            }
            const mixllm_epilogue ep = e.of(dev);
            if (rc == MIXLLM_OK)
                rc = mixed_linear_fp16_epilogue(&d, address(x), address(L.w4, dev), address(L.w8, dev), address(L.s4, dev), address(L.s8, dev),
                                                address(L.z4, dev), (const int32_t *)address(L.perm, dev), &ep, address(y, dev), address(ws, dev),
                                                (size_t)ws.numel(), stream);
        }
        return rc == MIXLLM_OK ? THPVariable_Wrap(std::move(y)) : PyLong_FromLong(rc);
    });
}

// activations as int8 codes [M][K] and fp16 scales [M][K / group]: the group
int32_t codes_and_scales(const at::Tensor &xq, const at::Tensor &xs, int64_t K)
{
    if (!xq.defined() || xq.dim() != 2 || xq.scalar_type() != at::kChar || xq.size(1) != K) throw Refused{"xq: int8, rows x inputs"};
    if (!xs.defined() || xs.dim() != 2 || xs.scalar_type() != at::kHalf || xs.size(0) != xq.size(0) || (xs.size(1) != 1 && xs.size(1) != K / MIXLLM_GROUP))
        throw Refused{"xs: fp16, one scale per row, or per row and group of 128"};
    return (int32_t)(xs.size(1) == 1 ? K : MIXLLM_GROUP);
}

// mixed_linear_epilogue(xq, xs, <layer>, bias, residual, activation, gated, out, workspace, stream) -> y, or a status
PyObject *py_mixed_linear_epilogue(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 19, [&]() -> PyObject * {
        const at::Tensor xq = tensor(a[0]), xs = tensor(a[1]);
        const Layer L(a + 2);
        const int32_t act_group = codes_and_scales(xq, xs, L.K);
        const int64_t M = xq.size(0);
        const Epilogue e(a + 12, M, L.N, 0);
        at::Tensor y = tensor(a[16]);
        const at::Tensor ws = tensor(a[17]);
        void *stream = PyLong_AsVoidPtr(a[18]);
        const at::Device dev = current(xq, "xq: an int8 matrix on the device");
        shaped(y, at::kHalf, {M, e.columns}, "out: fp16, tokens x outputs");
        if (!y.defined() && overrides_new_empty(a[0])) y = new_empty_in_python(a[0], M, e.columns, at::kHalf);
        int rc;
        {
            py::gil_scoped_release no_gil;
            if (!y.defined()) y = xq.new_empty({M, e.columns}, xq.options().dtype(at::kHalf));
            const mixllm_desc d{(int32_t)M, L.K, L.N, L.n8, MIXLLM_GROUP, act_group, L.w8_group};
            const mixllm_epilogue ep = e.of(dev);
            rc = mixed_linear_epilogue(&d, (const int8_t *)address(xq), address(xs, dev), address(L.w4, dev), address(L.w8, dev),
                                       address(L.s4, dev), address(L.s8, dev), address(L.z4, dev), (const int32_t *)address(L.perm, dev), &ep,
                                       address(y, dev), address(ws, dev), ws.defined() ? (size_t)ws.numel() : 0, stream);
        }
        return rc == MIXLLM_OK ? THPVariable_Wrap(std::move(y)) : PyLong_FromLong(rc);
    });
}

// route_experts(logits, top_k, score, bias, mask, groups, top_groups, group_score, renormalize, scale, stream)
// -> (ids, weights, offsets, rows, slots), or a status
PyObject *py_route_experts(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 11, [&]() -> PyObject * {
        const at::Tensor logits = tensor(a[0]);
        const at::Tensor bias = tensor(a[3]), mask = tensor(a[4]);
        if (!logits.defined() || logits.dim() != 2 || (logits.scalar_type() != at::kFloat && logits.scalar_type() != at::kHalf))
            throw Refused{"logits: fp16 or fp32, tokens x experts"};
        const at::Device dev = current(logits, "logits on the device");
        const int64_t T = logits.size(0), E = logits.size(1);
        const int64_t stride = T > 1 ? logits.stride(0) : std::max<int64_t>(E, 1);
        if ((E > 1 && logits.stride(1) != 1) || stride < E || stride > INT32_MAX) throw Refused{"logits: a token's experts next to each other"};
        shaped(bias, at::kFloat, {E}, "bias: fp32, one per expert");
        if (mask.defined() && mask.scalar_type() != at::kByte && mask.scalar_type() != at::kBool) throw Refused{"mask: bool or uint8, one per token"};
        shaped(mask, mask.defined() ? mask.scalar_type() : at::kByte, {T}, "mask: bool or uint8, one per token");
        mixllm_route_desc r{};
        r.T = (int32_t)std::min<int64_t>(T, INT32_MAX);
        r.E = (int32_t)std::min<int64_t>(E, INT32_MAX);
        r.top_k = number(a[1]);
        r.logits_fp16 = logits.scalar_type() == at::kHalf;
        r.logits_stride = (int32_t)stride;
        r.score = number(a[2]);
        r.groups = number(a[5]);
        r.top_groups = number(a[6]);
        r.group_score = number(a[7]);
        r.renormalize = truth(a[8]);
        r.scale = (float)PyFloat_AsDouble(a[9]);
        if (PyErr_Occurred()) throw python_error();
        void *stream = PyLong_AsVoidPtr(a[10]);
        if (r.top_k <= 0 || r.top_k > E) return PyLong_FromLong(MIXLLM_EINVAL);
        const int64_t k = r.top_k;
        at::Tensor out[5];
        if (overrides_new_empty(a[0])) {
            out[0] = new_empty_in_python(a[0], T, k, at::kInt);
            out[1] = new_empty_in_python(a[0], T, k, at::kFloat);
            out[2] = new_empty_in_python(a[0], py::make_tuple(E + 1), at::kInt);
            out[3] = new_empty_in_python(a[0], py::make_tuple(T * k), at::kInt);
            out[4] = new_empty_in_python(a[0], T, k, at::kInt);
        }
        int rc;
        {
            py::gil_scoped_release no_gil;
            if (!out[0].defined()) {
                const auto ints = logits.options().dtype(at::kInt);
                out[0] = at::empty({T, k}, ints);
                out[1] = at::empty({T, k}, logits.options().dtype(at::kFloat));
                out[2] = at::empty({E + 1}, ints);
                out[3] = at::empty({T * k}, ints);
                out[4] = at::empty({T, k}, ints);
            }
            const int64_t need = (int64_t)route_workspace(&r);
            at::Tensor ws;
            if (need) ws = at::empty({need}, logits.options().dtype(at::kByte));
            rc = route_experts(&r, T && E ? logits.data_ptr() : nullptr, (const float *)address(bias, dev), (const uint8_t *)address(mask, dev),
                               (int32_t *)address(out[0]), (float *)address(out[1]), (int32_t *)address(out[2]), (int32_t *)address(out[3]),
                               (int32_t *)address(out[4]), address(ws), (size_t)need, stream);
        }
        if (rc != MIXLLM_OK) return PyLong_FromLong(rc);
        const py::object all = py::reinterpret_steal<py::object>(PyTuple_New(5));
        if (!all) throw python_error();
        for (int i = 0; i < 5; ++i) {
            PyObject *t = THPVariable_Wrap(std::move(out[i]));
            if (!t) throw python_error();
            PyTuple_SET_ITEM(all.ptr(), i, t);
        }
        return py::object(all).release().ptr();
    });
}

// a route's list: int32 of n values
void list_of(const at::Tensor &t, int64_t n, const char *what)
{
    if (!t.defined() || t.scalar_type() != at::kInt || t.numel() != n) throw Refused{what};
}

// K, N, w8_group, E, table, n8 of the experts; offsets, rows, slots of the route; gather
struct Experts {
    int32_t K, N, w8_group, E, n8;
    at::Tensor table, offsets, rows, slots;
    bool gather;
    explicit Experts(PyObject *const *a)
        : K(number(a[0])), N(number(a[1])), w8_group(number(a[2])), E(number(a[3])), n8(number(a[5])), table(tensor(a[4])), offsets(tensor(a[6])),
          rows(tensor(a[7])), slots(tensor(a[8])), gather(truth(a[9]))
    {
        if (!table.defined() || table.nbytes() < experts_table_bytes(E)) throw Refused{"table: an entry for every expert"};
        list_of(offsets, (int64_t)E + 1, "the route and the layer agree in their experts");
        if (!slots.defined() || slots.dim() != 2 || slots.scalar_type() != at::kInt) throw Refused{"slots: int32, tokens x top_k"};
        list_of(rows, slots.numel(), "rows: int32, one per assignment");
    }
    // rows of the activations -> places
    int64_t places(int64_t M) const
    {
        if (M != (gather ? slots.size(0) : slots.numel())) throw Refused{"activations: a row per token (gather) or per assignment"};
        return slots.numel();
    }
};

// experts_linear_fp16(x, <experts>, act_group, bias, activation, gated, out, workspace, stream) -> y, or a status
// experts_linear(xq, xs, <experts>, bias, activation, gated, out, stream) -> y, or a status
template <bool FP16>
PyObject *py_experts_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, FP16 ? 18 : 17, [&]() -> PyObject * {
        const at::Tensor x = tensor(a[0]), xs = FP16 ? at::Tensor() : tensor(a[1]);
        const Experts L(a + (FP16 ? 1 : 2));
        PyObject *const *rest = a + 12;   // bias, activation, gated, out, (workspace,) stream
        if (FP16) half_matrix(x);
        const int32_t act_group = FP16 ? number(a[11]) : codes_and_scales(x, xs, L.K);
        if (x.size(1) != L.K) throw Refused{"x has as many columns as the layers have inputs"};
        const int64_t M = x.size(0), places = L.places(M);
        PyObject *const epilogue[4] = {rest[0], Py_None, rest[1], rest[2]};
        const Epilogue e(epilogue, places, L.N, L.E);
        at::Tensor y = tensor(rest[3]), ws = FP16 ? tensor(rest[4]) : at::Tensor();
        void *stream = PyLong_AsVoidPtr(rest[FP16 ? 5 : 4]);
        const at::Device dev = current(x, "activations on the device");
        shaped(y, at::kHalf, {places, e.columns}, "out: fp16, assignments x outputs");
        if (!y.defined() && overrides_new_empty(a[0])) y = new_empty_in_python(a[0], places, e.columns, at::kHalf);
        int rc;
        {
            py::gil_scoped_release no_gil;
            if (!y.defined()) y = at::empty({places, e.columns}, x.options().dtype(at::kHalf));
            const mixllm_desc d{(int32_t)M, L.K, L.N, L.n8, MIXLLM_GROUP, act_group, L.w8_group};
            const mixllm_epilogue ep = e.of(dev);
            const int32_t gather = L.gather ? (int32_t)L.slots.size(1) : 0;
            if (FP16) {
                if (!ws.defined()) ws = at::empty({(int64_t)experts_workspace(&d)}, x.options().dtype(at::kByte));
                rc = experts_linear_fp16(&d, L.E, address(L.table, dev), address(x), (const int32_t *)address(L.offsets, dev),
                                         (const int32_t *)address(L.rows, dev), gather, &ep, address(y, dev), address(ws, dev), (size_t)ws.numel(),
                                         stream);
            } else
                rc = experts_linear(&d, L.E, address(L.table, dev), (const int8_t *)address(x), address(xs, dev),
                                    (const int32_t *)address(L.offsets, dev), (const int32_t *)address(L.rows, dev), gather, &ep, address(y, dev),
                                    stream);
        }
        return rc == MIXLLM_OK ? THPVariable_Wrap(std::move(y)) : PyLong_FromLong(rc);
    });
}

// experts_combine(y, weights, slots, residual, out, stream) -> out, or a status
PyObject *py_experts_combine(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 6, [&]() -> PyObject * {
        const at::Tensor y = tensor(a[0]), weights = tensor(a[1]), slots = tensor(a[2]), residual = tensor(a[3]);
        at::Tensor out = tensor(a[4]);
        void *stream = PyLong_AsVoidPtr(a[5]);
        half_matrix(y);
        if (!slots.defined() || slots.dim() != 2 || slots.scalar_type() != at::kInt) throw Refused{"slots: int32, tokens x top_k"};
        if (!weights.defined()) throw Refused{"weights: fp32, tokens x top_k"};
        const int64_t T = slots.size(0), k = slots.size(1), N = y.size(1);
        shaped(weights, at::kFloat, {T, k}, "weights: fp32, tokens x top_k");
        shaped(residual, at::kHalf, {T, N}, "residual: fp16, of the result's shape");
        shaped(out, at::kHalf, {T, N}, "out: fp16, tokens x outputs");
        const at::Device dev = current(y, "y: an fp16 matrix on the device");
        if (!out.defined() && overrides_new_empty(a[0])) out = new_empty_in_python(a[0], T, N, at::kHalf);
        int rc;
        {
            py::gil_scoped_release no_gil;
            if (!out.defined()) out = at::empty({T, N}, y.options());
            rc = experts_combine((int32_t)T, (int32_t)k, (int32_t)N, (int32_t)y.size(0), address(y), (const float *)address(weights, dev),
                                 (const int32_t *)address(slots, dev), address(residual, dev), address(out, dev), stream);
        }
        return rc == MIXLLM_OK ? THPVariable_Wrap(std::move(out)) : PyLong_FromLong(rc);
    });
}

// bind(addresses of the library's functions, in the order below)
PyObject *py_bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return run(n, 13, [&]() -> PyObject * {
        auto take = [&](auto &f, int i) { f = (std::remove_reference_t<decltype(f)>)PyLong_AsVoidPtr(a[i]); };
        take(query_sizes, 0);
        take(quantize_activations, 1);
        take(mixed_linear_path, 2);
        take(mixed_linear_fp16, 3);
        take(mixed_linear_epilogue, 4);
        take(mixed_linear_fp16_epilogue, 5);
        take(route_workspace, 6);
        take(route_experts, 7);
        take(experts_workspace, 8);
        take(experts_linear, 9);
        take(experts_linear_fp16, 10);
        take(experts_combine, 11);
        take(experts_table_bytes, 12);
        Py_RETURN_NONE;
    });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)())py_bind, METH_FASTCALL, nullptr},
    {"linear_fp16", (PyCFunction)(void (*)())py_linear_fp16, METH_FASTCALL, nullptr},
    {"quantize_activations", (PyCFunction)(void (*)())py_quantize_activations, METH_FASTCALL, nullptr},
    {"mixed_linear", (PyCFunction)(void (*)())py_mixed_linear, METH_FASTCALL, nullptr},
    {"linear_fp16_epilogue", (PyCFunction)(void (*)())py_linear_fp16_epilogue, METH_FASTCALL, nullptr},
    {"mixed_linear_epilogue", (PyCFunction)(void (*)())py_mixed_linear_epilogue, METH_FASTCALL, nullptr},
    {"route_experts", (PyCFunction)(void (*)())py_route_experts, METH_FASTCALL, nullptr},
    {"experts_linear", (PyCFunction)(void (*)())py_experts_linear<false>, METH_FASTCALL, nullptr},
    {"experts_linear_fp16", (PyCFunction)(void (*)())py_experts_linear<true>, METH_FASTCALL, nullptr},
    {"experts_combine", (PyCFunction)(void (*)())py_experts_combine, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
