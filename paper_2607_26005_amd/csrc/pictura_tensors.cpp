// Reads torch tensors for the binding: their device addresses, after every check that
// keeps a kernel inside its buffers.  In Python those checks take 0.5 us a vector and
// some 4 us an optimizer's tensor (29 tensors of the policy: 115 us a step, ten times
// the step's kernels); here 0.1 us.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <sstream>
#include <stdexcept>

namespace {

// pictura_adamw_tensor (include/pictura.h)
struct Row {
    uint64_t param, grad, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale;
    int64_t n;
    int32_t param_dtype, grad_dtype;
};
static_assert(sizeof(Row) == 64, "one row of the table");

constexpr int64_t kBlock = 256;   // PICTURA_ADAMW_BLOCK

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};

template <class... A>
[[noreturn]] void refuse(const A&... a)
{
    std::ostringstream s;
    (void)(s << ... << a);
    throw Refused(s.str());
}

const at::Tensor& tensor(PyObject* o, const char* what, Py_ssize_t i)
{
    if (!THPVariable_Check(o)) refuse(what, " ", i, ": expected a torch tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

int32_t dtype_code(const at::Tensor& t, const char* what)
{
    switch (t.scalar_type()) {
    case at::kFloat: return 0;
    case at::kBFloat16: return 1;
    case at::kHalf: return 2;
    default: refuse(what, ": dtype ", t.scalar_type(), ", expected float32, bfloat16 or float16");
    }
}

// Address of one of a parameter's moments or scales.
uint64_t held(PyObject* state, const char* key, at::ScalarType kind, int64_t count, const at::Device& dev, Py_ssize_t i)
{
    PyObject* o = PyDict_GetItemString(state, key);   // borrowed
    if (!o || !THPVariable_Check(o)) refuse("state of parameter ", i, ": no tensor ", key);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || t.scalar_type() != kind || t.numel() != count || t.device() != dev || !t.is_contiguous())
        refuse("state of parameter ", i, ": ", key, " is ", t.scalar_type(), " of ", t.numel(), " elements on ", t.device(),
               ", expected ", kind, " of ", count, " on ", dev);
    return (uint64_t)(uintptr_t)t.data_ptr();
}

// fill(params, grads, states, bits, table, steps) -> (rows, index of the first parameter
// that took one, or -1): all that did are on that one's device.  None: a state that a
// row needs has not begun (no "step").  grads: a list (None: no
// gradient), True for the parameters' own, False for none needed; a parameter without
// a gradient where one is needed takes no row.  states: dicts.  steps: int64, one for
// each row.  Gradients mean a step, which writes the parameters of all rows: their
// version goes up, so that autograd refuses a graph that saved them before.
PyObject* fill(PyObject*, PyObject* args)
{
    PyObject *params, *grads, *states;
    int bits;
    Py_buffer table, steps;
    if (!PyArg_ParseTuple(args, "O!OO!iw*w*", &PyList_Type, &params, &grads, &PyList_Type, &states, &bits, &table, &steps))
        return nullptr;
    PyObject* result = nullptr;
    try {
        const Py_ssize_t count = PyList_GET_SIZE(params);
        const bool listed = PyList_Check(grads), own = grads == Py_True;
        if (PyList_GET_SIZE(states) != count || (listed && PyList_GET_SIZE(grads) != count) ||
            table.len < count * (Py_ssize_t)sizeof(Row) || steps.len < count * (Py_ssize_t)sizeof(int64_t))
            refuse("lists of different lengths");
        Row* out = static_cast<Row*>(table.buf);
        int64_t* step = static_cast<int64_t*>(steps.buf);
        Py_ssize_t rows = 0, first = -1;
        bool begun = true;
        at::Device dev(at::kCPU);
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor& p = tensor(PyList_GET_ITEM(params, i), "parameter", i);
            Row r{};
            const at::Tensor* g = nullptr;
            if (listed) {
                PyObject* o = PyList_GET_ITEM(grads, i);
                if (o == Py_None) continue;
                g = &tensor(o, "gradient", i);
            } else if (own) {
                g = &p.grad();
                if (!g->defined()) continue;
            }
            if (rows == 0) {
                dev = p.device();
                first = i;
            }
            if (p.device() != dev) refuse("parameter ", i, ": on ", p.device(), ", others on ", dev);
            if (p.layout() != at::kStrided || !p.is_contiguous() || p.is_neg()) refuse("parameter ", i, ": tensor is not contiguous");
            r.param_dtype = dtype_code(p, "parameter");
            r.n = p.numel();
            r.param = (uint64_t)(uintptr_t)p.data_ptr();
            if (g) {
                if (g->layout() != at::kStrided || g->device() != dev || g->sizes() != p.sizes() || !g->is_contiguous() || g->is_neg())
                    refuse("gradient ", i, ": ", g->scalar_type(), " ", g->sizes(), " on ", g->device(),
                           ", expected a contiguous tensor of the parameter's shape ", p.sizes(), " on ", dev);
                r.grad_dtype = dtype_code(*g, "gradient");
                r.grad = (uint64_t)(uintptr_t)g->data_ptr();
            }
            PyObject* s = PyList_GET_ITEM(states, i);
            if (!PyDict_Check(s)) refuse("state of parameter ", i, ": no state");
            PyObject* k = PyDict_GetItemString(s, "step");
            if (!k) {
                begun = false;
                break;
            }
            const bool small = bits == 8;
            r.exp_avg = held(s, "exp_avg", small ? at::kChar : at::kFloat, r.n, dev, i);
            r.exp_avg_sq = held(s, "exp_avg_sq", small ? at::kByte : at::kFloat, r.n, dev, i);
            if (small) {
                const int64_t blocks = (r.n + kBlock - 1) / kBlock;
                r.exp_avg_scale = held(s, "exp_avg_scale", at::kFloat, blocks, dev, i);
                r.exp_avg_sq_scale = held(s, "exp_avg_sq_scale", at::kFloat, blocks, dev, i);
            }
            const long long at_step = PyLong_Check(k) ? PyLong_AsLongLong(k) : -1;
            if (at_step < 0) {
                PyErr_Clear();
                refuse("state of parameter ", i, ": step is not a whole number");
            }
            step[rows] = at_step;
            out[rows++] = r;
        }
        for (Py_ssize_t i = first; begun && rows > 0 && (listed || own) && i < count; ++i) {
            const at::Tensor& p = THPVariable_Unpack(PyList_GET_ITEM(params, i));
            const bool steps_too = listed ? PyList_GET_ITEM(grads, i) != Py_None : p.grad().defined();
            if (steps_too && !p.is_inference()) p.unsafeGetTensorImpl()->bump_version();   // (those have none)
        }
        result = begun ? Py_BuildValue("nn", rows, first) : Py_NewRef(Py_None);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
    }
    PyBuffer_Release(&table);
    PyBuffer_Release(&steps);
    return result;
}

const char* type_name(at::ScalarType k)
{
    return k == at::kFloat ? "float32" : k == at::kLong ? "int64" : "int32";
}

// vectors(like, count, (name, kind, tensor), ...) -> addresses.  Each tensor is a
// contiguous vector of `count` elements on the device of `like`, kind "f" float32, "l"
// int64 or "i" int32; None gives 0.
PyObject* vectors(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n < 2 || (n - 2) % 3 || !THPVariable_Check(args[0]) || !PyLong_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "vectors(like, count, name, kind, tensor, ...)");
        return nullptr;
    }
    PyObject* result = PyTuple_New((n - 2) / 3);
    if (!result) return nullptr;
    try {
        const at::Device dev = THPVariable_Unpack(args[0]).device();
        const int64_t count = PyLong_AsLongLong(args[1]);
        for (Py_ssize_t k = 2; k < n; k += 3) {
            const char* name = PyUnicode_AsUTF8(args[k]);
            const char* code = PyUnicode_AsUTF8(args[k + 1]);
            if (!name || !code) refuse("a name is no text");
            const at::ScalarType kind = *code == 'f' ? at::kFloat : *code == 'l' ? at::kLong : at::kInt;
            uint64_t at = 0;
            if (args[k + 2] != Py_None) {
                if (!THPVariable_Check(args[k + 2]))
                    refuse(name, ": expected a torch tensor on the HIP device, got ", Py_TYPE(args[k + 2])->tp_name);
                const at::Tensor& t = THPVariable_Unpack(args[k + 2]);
                if (t.device() != dev) refuse(name, ": tensor on ", t.device(), ", the logits are on ", dev);
                if (t.scalar_type() != kind) refuse(name, ": dtype ", t.scalar_type(), ", expected ", type_name(kind));
                if (t.dim() != 1 || t.size(0) != count) refuse(name, ": shape ", t.sizes(), ", expected [", count, "]");
                if (t.layout() != at::kStrided || !t.is_contiguous() || t.is_neg()) refuse(name, ": tensor is not contiguous");
                at = (uint64_t)(uintptr_t)t.data_ptr();
            }
            PyObject* o = PyLong_FromUnsignedLongLong(at);
            if (!o) refuse("out of memory");
            PyTuple_SET_ITEM(result, (k - 2) / 3, o);
        }
        return result;
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
    }
    Py_DECREF(result);
    return nullptr;
}

// outputs(tensors, params) -> bytes: the addresses of contiguous fp32 tensors of the
// parameters' sizes.
PyObject* outputs(PyObject*, PyObject* args)
{
    PyObject *tensors, *params;
    if (!PyArg_ParseTuple(args, "O!O!", &PyList_Type, &tensors, &PyList_Type, &params)) return nullptr;
    const Py_ssize_t count = PyList_GET_SIZE(params);
    PyObject* result = PyBytes_FromStringAndSize(nullptr, count * (Py_ssize_t)sizeof(uint64_t));
    if (!result) return nullptr;
    try {
        if (PyList_GET_SIZE(tensors) != count) refuse("out: ", PyList_GET_SIZE(tensors), " tensors for ", count, " parameters");
        uint64_t* to = reinterpret_cast<uint64_t*>(PyBytes_AS_STRING(result));
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor& t = tensor(PyList_GET_ITEM(tensors, i), "out", i);
            const at::Tensor& p = tensor(PyList_GET_ITEM(params, i), "parameter", i);
            if (t.layout() != at::kStrided || t.scalar_type() != at::kFloat || t.numel() != p.numel() || !t.is_contiguous() ||
                t.device() != p.device())
                refuse("out ", i, ": ", t.scalar_type(), " of ", t.numel(), " elements, expected float32 of ", p.numel());
            to[i] = (uint64_t)(uintptr_t)t.data_ptr();
        }
        return result;
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
    }
    Py_DECREF(result);
    return nullptr;
}

PyMethodDef methods[] = {{"outputs", outputs, METH_VARARGS, "Addresses of fp32 tensors of the parameters' sizes."},
                         {"vectors", (PyCFunction)(void (*)())vectors, METH_FASTCALL, "Addresses of vectors of one length."},
                         {"fill", fill, METH_VARARGS, "Fill a table of pictura_adamw_tensor from lists of tensors."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
