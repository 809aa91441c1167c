// The calls of the operators around a language model's layers on torch's tensors, as an extension module of Python.
//
// Small calls are bound by what the host does before a kernel starts.  Through ctypes the host took 40 us for the gradients of a block's norms (sixteen operands, two launches of 3.7 us each),
// 17.5 for its forward call and 9.5 for a lookup; here 14, 5.9 and 4.3.  The module checks tensors and allocates outputs and workspaces; everything else is checked by the C entry points, whose
// addresses it is given.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <string>

#include "../../include/netmax.h"

namespace {

PyObject *g_error, *g_stream;                      // NetmaxError; torch's function from a device's number to the handle of its current stream
struct {
    decltype(&netmax_last_error) last_error;
    decltype(&netmax_embed) embed;
    decltype(&netmax_embed_grad_workspace) embed_grad_workspace;
    decltype(&netmax_embed_grad) embed_grad;
    decltype(&netmax_block_norm) block_norm;
    decltype(&netmax_block_norm_grad_workspace) block_norm_grad_workspace;
    decltype(&netmax_block_norm_grad) block_norm_grad;
    decltype(&netmax_grad_norm_workspace) grad_norm_workspace;
    decltype(&netmax_grad_norm) grad_norm;
    decltype(&netmax_clip_grads) clip_grads;
} lib;

// What leads out of a call to the place that raises it in Python.
struct Refusal { int code; std::string text; };
[[noreturn]] void refuse(const char *format, ...)
{
    char text[400];
    va_list args;
    va_start(args, format);
    vsnprintf(text, sizeof text, format, args);
    va_end(args);
    throw Refusal{NETMAX_EINVAL, text};
}
struct PythonError { };                            // one that Python knows already

std::string written(at::IntArrayRef sizes)
{
    std::string s = "(";
    for (size_t k = 0; k < sizes.size(); ++k) s += (k ? ", " : "") + std::to_string(sizes[k]);
    return s + (sizes.size() == 1 ? ",)" : ")");
}

int32_t dtype_of(const at::Tensor &t) { return t.scalar_type() == at::kBFloat16 ? NETMAX_BF16 : NETMAX_F32; }
bool rows_are_dense(const at::Tensor &t) { return t.dim() == 0 || t.size(-1) <= 1 || t.stride(-1) == 1; }

void no_graph(const char *name, const at::Tensor &t)
{
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse("%s requires a gradient, which this call does not record: call it under torch.no_grad() or with a detached tensor", name);
}

// The tensor that says device, type and sizes: float32 or bfloat16, two or three dimensions.
const at::Tensor &leading(const char *name, PyObject *o)
{
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) refuse("%s must be a tensor on the GPU", name);
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != 2 && t.dim() != 3) refuse("%s has %d dimensions", name, (int)t.dim());
    if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) refuse("%s is %s: float32 or bfloat16 is needed", name, toString(t.scalar_type()));
    if (!rows_are_dense(t)) refuse("the values of a row of %s must lie next to each other", name);
    no_graph(name, t);
    return t;
}

const at::Tensor &checked(const char *name, PyObject *o, const at::Tensor &like, at::IntArrayRef sizes, at::ScalarType type)
{
    if (!THPVariable_Check(o)) refuse("%s must be a tensor", name);
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.device() != like.device()) refuse("%s is on %s, not on %s", name, t.device().str().c_str(), like.device().str().c_str());
    if (t.scalar_type() != type) refuse("%s is %s, not %s", name, toString(t.scalar_type()), toString(type));
    if (t.sizes() != sizes) refuse("%s has the shape %s, not %s", name, written(t.sizes()).c_str(), written(sizes).c_str());
    if (!rows_are_dense(t)) refuse("the values of a row of %s must lie next to each other", name);
    no_graph(name, t);
    return t;
}

// Tensors made in inference mode have no version.
void changed(PyObject *o)
{
    if (o && o != Py_None && !THPVariable_Unpack(o).is_inference()) THPVariable_Unpack(o).unsafeGetTensorImpl()->bump_version();
}

int64_t row_distance(const at::Tensor &t) { return t.stride(t.dim() - 2); }
int64_t batch_distance(const at::Tensor &t) { return t.dim() == 3 ? t.stride(0) : 0; }
netmax_span rows_span(const at::Tensor &t) { return {t.data_ptr(), row_distance(t), batch_distance(t)}; }
netmax_span vector_span(const at::Tensor &t) { return {t.data_ptr(), 0, t.dim() == 2 ? t.stride(0) : 0}; }

// Calls of one device: it is the current one meanwhile, and its current stream takes the work.
struct Place {
    c10::DeviceGuard guard;
    c10::TensorOptions options;
    explicit Place(const at::Tensor &t) : guard(t.device()), options(t.options().requires_grad(false)) { }
    void *stream() const
    {
        PyObject *index = PyLong_FromLong(guard.current_device().index()), *handle = index ? PyObject_CallOneArg(g_stream, index) : nullptr;
        Py_XDECREF(index);
        if (!handle) throw PythonError{};
        void *s = PyLong_AsVoidPtr(handle);
        Py_DECREF(handle);
        return s;
    }
    at::Tensor empty(at::IntArrayRef sizes) const { return at::empty(sizes, options); }
    at::Tensor workspace(int64_t bytes) const
    {
        if (bytes < 0) throw Refusal{NETMAX_EINVAL, lib.last_error(nullptr)};
        return bytes ? at::empty({bytes}, options.dtype(at::kByte)) : at::Tensor();
    }
};
void *address(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
void check(int code)
{
    if (code != NETMAX_OK) throw Refusal{code, lib.last_error(nullptr)};
}

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
    return v;
}
int64_t whole(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError{};
    return v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError{};
    return v;
}
PyObject *new_reference(PyObject *o) { Py_INCREF(o); return o; }
PyObject *wrapped(const at::Tensor &t) { return t.defined() ? THPVariable_Wrap(t) : new_reference(Py_None); }

template <class Body> PyObject *guarded(Py_ssize_t given, Py_ssize_t needed, const Body &body) noexcept
{
    if (given != needed) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", given, needed);
        return nullptr;
    }
    try {
        return body();
    } catch (const Refusal &r) {
        PyObject *e = PyObject_CallFunction(g_error, "is", r.code, r.text.c_str());
        if (e) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
    } catch (const PythonError &) {
    } catch (...) {                                // torch's own, out of memory among them
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// ---- embedding -------------------------------------------------------------------------------------------------------

// Token ids for rows of a tensor of two dimensions, or three.
const at::Tensor &ids_for(PyObject *o, const at::Tensor &like)
{
    const int64_t lead = like.dim() - 2;
    if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() != 1 + lead) refuse("tokens must have one dimension for one table, two for a batch of them");
    const at::Tensor &t = THPVariable_Unpack(o);
    return lead ? checked("tokens", o, like, {like.size(0), t.size(1)}, at::kInt) : checked("tokens", o, like, {t.size(0)}, at::kInt);
}

c10::SmallVector<int64_t, 3> sizes_of(const at::Tensor &like, int64_t rows, int64_t width)
{
    c10::SmallVector<int64_t, 3> s;
    if (like.dim() == 3) s.push_back(like.size(0));
    s.push_back(rows);
    s.push_back(width);
    return s;
}

// tokens, table, scale, y
PyObject *embed(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 4, [&] {
        const at::Tensor &table = leading("table", a[1]), &ids = ids_for(a[0], table);
        const Place place(table);
        const auto sizes = sizes_of(table, ids.size(-1), table.size(-1));
        const bool given = a[3] != Py_None;
        const at::Tensor y = given ? checked("y", a[3], table, sizes, table.scalar_type()) : place.empty(sizes);
        const netmax_embed_shape s{table.dim() == 3 ? table.size(0) : 1, ids.size(-1), table.size(-2), table.size(-1), dtype_of(table), 0, (float)number(a[2]),
                                   ids.dim() == 2 ? ids.stride(0) : 0, row_distance(table), batch_distance(table), row_distance(y), batch_distance(y)};
        check(lib.embed(&s, (const int32_t *)ids.data_ptr(), table.data_ptr(), y.data_ptr(), place.stream()));
        changed(a[3]);
        return given ? new_reference(a[3]) : wrapped(y);
    });
}

// dy, tokens, vocab, scale, accumulate, dtable
PyObject *embed_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const at::Tensor &dy = leading("dy", a[0]), &ids = ids_for(a[1], dy);
        const bool given = a[5] != Py_None, accumulate = truth(a[4]);
        if (dy.size(-2) != ids.size(-1)) refuse("dy has %lld rows for %lld tokens", (long long)dy.size(-2), (long long)ids.size(-1));
        if (given && (!THPVariable_Check(a[5]) || THPVariable_Unpack(a[5]).dim() != dy.dim())) refuse("dtable must have as many dimensions as dy");
        if (!given && accumulate) refuse("accumulate needs dtable");
        if (!given && a[2] == Py_None) refuse("vocab or dtable is needed");
        const int64_t vocab = a[2] != Py_None ? whole(a[2]) : THPVariable_Unpack(a[5]).size(-2);
        if (vocab < 0) refuse("vocab is negative");
        const Place place(dy);
        const auto sizes = sizes_of(dy, vocab, dy.size(-1));
        const netmax_embed_shape sized{dy.dim() == 3 ? dy.size(0) : 1, ids.size(-1), vocab, dy.size(-1), dtype_of(dy), accumulate, (float)number(a[3]), ids.dim() == 2 ? ids.stride(0) : 0,
                                       0, 0, row_distance(dy), batch_distance(dy)};
        const at::Tensor work = place.workspace(lib.embed_grad_workspace(&sized));          // refuses sizes before a table is allocated
        const at::Tensor dtable = given ? checked("dtable", a[5], dy, sizes, dy.scalar_type()) : place.empty(sizes);
        netmax_embed_shape s = sized;
        s.ldt = row_distance(dtable);
        s.st = batch_distance(dtable);
        check(lib.embed_grad(&s, (const int32_t *)ids.data_ptr(), dy.data_ptr(), dtable.data_ptr(), address(work), work.defined() ? work.numel() : 0, place.stream()));
        changed(a[5]);
        return given ? new_reference(a[5]) : wrapped(dtable);
    });
}

// ---- norms of a block ------------------------------------------------------------------------------------------------

// x, f, gate, post_gain, post_bias, pre_gain, pre_bias; norm, post, pre, gate_act, x_scale, f_scale, eps
constexpr int OPERANDS = 7, OPTIONS = 7;
struct Norm {
    const at::Tensor &x;
    netmax_block_norm_shape shape;
    netmax_block_norm_data data{};
    c10::SmallVector<int64_t, 2> vector;           // sizes of a gain
    bool gate_rows;

    netmax_span rows(const char *name, PyObject *o) const { return o == Py_None ? netmax_span{} : rows_span(checked(name, o, x, x.sizes(), x.scalar_type())); }
    netmax_span channels(const char *name, PyObject *o) const { return o == Py_None ? netmax_span{} : vector_span(checked(name, o, x, vector, x.scalar_type())); }
    netmax_span gate(const char *name, PyObject *o) const { return gate_rows ? rows(name, o) : channels(name, o); }

    Norm(PyObject *const *a, PyObject *const *o) : x(leading("x", a[0]))
    {
        if (x.dim() == 3) vector.push_back(x.size(0));
        vector.push_back(x.size(-1));
        gate_rows = THPVariable_Check(a[2]) && THPVariable_Unpack(a[2]).dim() == x.dim();
        shape = {x.dim() == 3 ? x.size(0) : 1, x.size(-2), x.size(-1), dtype_of(x), (int32_t)whole(o[0]), (int32_t)whole(o[3]), gate_rows, truth(o[1]), truth(o[2]),
                 (float)number(o[4]), (float)number(o[5]), (float)number(o[6])};
        data.x = rows_span(x);
        data.f = rows("f", a[1]);
        data.gate = gate("gate", a[2]);
        data.post_gain = channels("post_gain", a[3]);
        data.post_bias = channels("post_bias", a[4]);
        data.pre_gain = channels("pre_gain", a[5]);
        data.pre_bias = channels("pre_bias", a[6]);
    }
};

// An output: what is given, or allocated if it is needed.
struct Output {
    PyObject *given;
    at::Tensor made;
    PyObject *result() const { return given != Py_None ? new_reference(given) : wrapped(made); }
};
netmax_span filled(Output &out, PyObject *given, bool needed, bool is_rows, const char *name, const Norm &n, const Place &place)
{
    out.given = given;
    if (given != Py_None) return is_rows ? n.rows(name, given) : n.channels(name, given);
    if (!needed) return netmax_span{};
    out.made = is_rows ? place.empty(n.x.sizes()) : place.empty(n.vector);
    return is_rows ? rows_span(out.made) : vector_span(out.made);
}

PyObject *tuple_of(Output *outputs, int n)
{
    PyObject *t = PyTuple_New(n);
    for (int k = 0; t && k < n; ++k) {
        PyObject *o = outputs[k].result();
        if (!o) {
            Py_DECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, k, o);
        changed(outputs[k].given);
    }
    return t;
}

// operands, options; need_h, h, y
PyObject *block_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, OPERANDS + OPTIONS + 3, [&] {
        Norm norm(a, a + OPERANDS);
        PyObject *const *o = a + OPERANDS + OPTIONS;
        const Place place(norm.x);
        Output out[2];
        norm.data.h = filled(out[0], o[1], a[1] != Py_None && truth(o[0]), true, "h", norm, place);
        norm.data.y = filled(out[1], o[2], norm.shape.pre, true, "y", norm, place);
        check(lib.block_norm(&norm.shape, &norm.data, place.stream()));
        return tuple_of(out, 2);
    });
}

// dy, dh; operands, options; need_input, need_params; dx, df, dgate, dpost_gain, dpost_bias, dpre_gain, dpre_bias
PyObject *block_norm_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 2 + OPERANDS + OPTIONS + 2 + OPERANDS, [&] {
        PyObject *const *in = a + 2, *const *o = in + OPERANDS + OPTIONS;
        const Norm norm(in, in + OPERANDS);
        const Place place(norm.x);
        const bool input = truth(o[0]), params = truth(o[1]);
        netmax_block_norm_grads g{};
        g.dy = norm.rows("dy", a[0]);
        g.dh = norm.rows("dh", a[1]);
        Output out[OPERANDS];
        static const char *const names[OPERANDS] = {"dx", "df", "dgate", "dpost_gain", "dpost_bias", "dpre_gain", "dpre_bias"};
        netmax_span *const spans[OPERANDS] = {&g.dx, &g.df, &g.dgate, &g.dpost_gain, &g.dpost_bias, &g.dpre_gain, &g.dpre_bias};
        for (int k = 0; k < OPERANDS; ++k) {
            const bool is_rows = k < 2 || (k == 2 && norm.gate_rows);
            *spans[k] = filled(out[k], o[2 + k], in[k] != Py_None && (is_rows ? input : params), is_rows, names[k], norm, place);
        }
        const at::Tensor work = place.workspace(lib.block_norm_grad_workspace(&norm.shape, &norm.data, &g));
        check(lib.block_norm_grad(&norm.shape, &norm.data, &g, address(work), work.defined() ? work.numel() : 0, place.stream()));
        return tuple_of(out, OPERANDS);
    });
}

// ---- clipping --------------------------------------------------------------------------------------------------------

// Whether a tensor lies as it did when its list was laid out, from `at` on: address, type, dimensions, sizes and strides.  What is behind is that of the next one.
void check_laid_out(const at::Tensor &t, const int64_t *&at, const int64_t *end)
{
    constexpr const char *CHANGED = "a gradient has changed its sizes, strides or type since the list was laid out";
    if (end - at < 3 || end - at - 3 < 2 * at[2]) refuse("a list of gradients that was not laid out");
    if ((int64_t)t.data_ptr() != at[0]) refuse("a gradient has moved since the list was laid out");
    const int64_t n = t.dim();
    if ((t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) || dtype_of(t) != at[1] || n != at[2]) refuse("%s", CHANGED);
    at += 3;
    if (t.sizes() != at::IntArrayRef(at, n) || t.strides() != at::IntArrayRef(at + n, n)) refuse("%s", CHANGED);
    at += 2 * n;
}

// tensors, outputs, how they lie as bytes; entries (address of netmax_gradient[]), models, whether there is a batch; max_norm or None
PyObject *clip(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        if (!PyTuple_Check(a[0]) || !PyTuple_Check(a[1]) || !PyBytes_Check(a[2])) refuse("a list of gradients that was not laid out");
        const Py_ssize_t count = PyTuple_GET_SIZE(a[0]);
        if (count < 1 || PyTuple_GET_SIZE(a[1]) != count) refuse("a list of gradients that has changed since it was laid out");
        const int64_t *at = (const int64_t *)PyBytes_AS_STRING(a[2]), *const end = at + PyBytes_GET_SIZE(a[2]) / (Py_ssize_t)sizeof(int64_t);
        for (int side = 0; side < 2; ++side)
            for (Py_ssize_t k = 0; k < count; ++k) {
                PyObject *o = PyTuple_GET_ITEM(a[side], k);
                if (!THPVariable_Check(o)) refuse("a gradient must be a tensor");
                const at::Tensor &t = THPVariable_Unpack(o);
                check_laid_out(t, at, end);
                no_graph("a gradient", t);
            }
        if (at != end) refuse("a list of gradients that has changed since it was laid out");
        const at::Tensor &first = THPVariable_Unpack(PyTuple_GET_ITEM(a[0], 0));
        const netmax_gradient *entries = (const netmax_gradient *)PyLong_AsVoidPtr(a[3]);
        const int64_t models = whole(a[4]);
        const Place place(first);
        const at::Tensor norm = truth(a[5]) ? at::empty({models}, place.options.dtype(at::kFloat)) : at::empty({}, place.options.dtype(at::kFloat));
        const at::Tensor work = place.workspace(lib.grad_norm_workspace(models, count, entries));
        const int64_t bytes = work.defined() ? work.numel() : 0;
        if (a[6] == Py_None) {
            check(lib.grad_norm(models, count, entries, (float *)norm.data_ptr(), address(work), bytes, place.stream()));
        } else {
            check(lib.clip_grads(models, count, entries, (float)number(a[6]), (float *)norm.data_ptr(), address(work), bytes, place.stream()));
            for (Py_ssize_t k = 0; k < count; ++k) changed(PyTuple_GET_ITEM(a[1], k));
        }
        return wrapped(norm);
    });
}

// NetmaxError, the function for streams, the addresses of the entry points in the order of `lib`
PyObject *setup(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        void *at[sizeof lib / sizeof(void *)];
        if (!PyTuple_Check(a[2]) || PyTuple_GET_SIZE(a[2]) != (Py_ssize_t)(sizeof lib / sizeof(void *))) refuse("as many addresses as entry points");
        for (size_t k = 0; k < sizeof lib / sizeof(void *); ++k) at[k] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[2], k));
        if (PyErr_Occurred()) throw PythonError{};
        memcpy(&lib, at, sizeof lib);
        g_error = new_reference(a[0]);
        g_stream = new_reference(a[1]);
        return new_reference(Py_None);
    });
}

#define METHOD(name) {#name, (PyCFunction)(void *)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(setup), METHOD(embed), METHOD(embed_grad), METHOD(block_norm), METHOD(block_norm_grad), METHOD(clip), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lm_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lm_calls() { return PyModule_Create(&module); }
