// Calls of the text model's operators from Python, on PyTorch tensors: what text.py's classes do on every call, in one step.
// A call of few tokens is bound by the host: of the 6.3 us that a lookup through ctypes took, the launch is 2.75, and checks, shapes
// and the allocation of the output in Python were 2.9; here they are 1.0.  Checks and allocation only: the operators are the
// library's, reached through addresses that text.py passes to bind().
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>

#include "../../include/sparse_conv.h"

namespace {

decltype(&sparse_conv_embed) embed = nullptr;
decltype(&sparse_conv_embed_backward_workspace) embed_backward_workspace = nullptr;
decltype(&sparse_conv_embed_backward) embed_backward = nullptr;
decltype(&sparse_conv_int8_linear_workspace) int8_linear_workspace = nullptr;
decltype(&sparse_conv_int8_linear) int8_linear = nullptr;

// SC_* of a floating-point type, -1 for any other.
int type_of(at::ScalarType t)
{
    return t == at::kFloat ? SC_F32 : t == at::kHalf ? SC_F16 : t == at::kBFloat16 ? SC_BF16 : -1;
}

// What ends in a ValueError.
struct Refused {
    const char* what;
};
void require(bool holds, const char* what)
{
    if (!holds) throw Refused{what};
}

const at::Tensor& tensor(PyObject* o, const char* what)
{
    require(THPVariable_Check(o), what);
    return THPVariable_Unpack(o);
}

// A status other than SC_OK goes back as a number (text.py raises the library's error from it).  given: `out` is the caller's, whose
// version counts what is written into it (autograd refuses to read what it saved once that has changed).
PyObject* result(int rc, const at::Tensor& out, bool given)
{
    if (given && !out.is_inference()) out.unsafeGetTensorImpl()->bump_version();
    return rc == SC_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
}

// Scratch memory of the current device and stream (text.py calls with the tensors' device as the current one), as at::empty gets it, but
// without a tensor around it.
c10::DataPtr workspace(long long bytes) { return bytes > 0 ? c10::GetAllocator(c10::DeviceType::CUDA)->allocate((size_t)bytes) : c10::DataPtr(); }

// The truth of an argument.
bool is_true(PyObject* o)
{
    const int t = PyObject_IsTrue(o);
    if (t < 0) PyErr_Clear();
    require(t >= 0, "a truth value is expected");
    return t != 0;
}

// torch.OutOfMemoryError, as every other allocation of the caller's raises it.
void set_out_of_memory(const char* what)
{
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    if (type) PyErr_SetString(type, what);
    Py_XDECREF(type);
    Py_XDECREF(torch);
}

template <class F>
PyObject* guarded(F&& f)
{
    try {
        return f();
    } catch (const Refused& r) {
        PyErr_SetString(PyExc_ValueError, r.what);
    } catch (const c10::OutOfMemoryError& e) {
        set_out_of_memory(e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

bool all_numbers(PyObject* const* args, Py_ssize_t from, Py_ssize_t to)
{
    for (Py_ssize_t i = from; i < to; ++i)
        if (!PyLong_Check(args[i])) return false;
    return true;
}

// bind(embed, embed_backward_workspace, embed_backward, int8_linear_workspace, int8_linear): addresses of the library's functions.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    if (count != 5 || !all_numbers(args, 0, 5)) {
        PyErr_SetString(PyExc_TypeError, "five addresses");
        return nullptr;
    }
    void* p[5];
    for (int i = 0; i < 5; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    embed = reinterpret_cast<decltype(embed)>(p[0]);
    embed_backward_workspace = reinterpret_cast<decltype(embed_backward_workspace)>(p[1]);
    embed_backward = reinterpret_cast<decltype(embed_backward)>(p[2]);
    int8_linear_workspace = reinterpret_cast<decltype(int8_linear_workspace)>(p[3]);
    int8_linear = reinterpret_cast<decltype(int8_linear)>(p[4]);
    Py_RETURN_NONE;
}

struct Sentences {
    int count, words;
    unsigned flags;
};

Sentences sentences_of(const at::Tensor& tokens, const at::Tensor& table, bool channels_first)
{
    const at::ScalarType t = tokens.scalar_type();
    require((t == at::kLong || t == at::kInt) && tokens.is_contiguous() && tokens.device() == table.device() && (!channels_first || tokens.dim() == 2),
            "tokens must be a contiguous tensor of 32- or 64-bit integers on the table's device ([sentences][words] for channels_first)");
    require(tokens.numel() < (1ll << 31), "2^31 tokens or more");
    const unsigned flags = t == at::kLong ? SC_EMBED_TOKENS_64 : 0u;
    if (channels_first) return {(int)tokens.size(0), (int)tokens.size(1), flags | SC_EMBED_CHANNELS_FIRST};
    return {1, (int)tokens.numel(), flags};
}

// Shape of the vectors of `tokens`.
c10::SmallVector<int64_t, 5> vectors_of(const at::Tensor& tokens, int64_t dim, bool channels_first)
{
    if (channels_first) return {tokens.size(0), dim, 1, tokens.size(1)};
    c10::SmallVector<int64_t, 5> shape(tokens.sizes().begin(), tokens.sizes().end());
    shape.push_back(dim);
    return shape;
}

void require_table(const at::Tensor& table)
{
    require(table.is_cuda() && type_of(table.scalar_type()) >= 0 && table.dim() == 2 && table.is_contiguous() && table.size(0) > 0 && table.size(1) > 0 &&
                table.size(1) < (1ll << 31),
            "table must be a contiguous CUDA tensor [vocab][dim] of fp32, binary16 or bfloat16");
}

// forward(table, tokens, out or None, channels_first, scale, stream)
PyObject* py_embed(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        require(embed, "not bound");
        require(count == 6 && PyFloat_Check(args[4]) && PyLong_Check(args[5]), "bad arguments");
        const at::Tensor& table = tensor(args[0], "table must be a tensor");
        const at::Tensor& tokens = tensor(args[1], "tokens must be a tensor");
        const bool first = is_true(args[3]);
        require_table(table);
        const Sentences s = sentences_of(tokens, table, first);
        const auto shape = vectors_of(tokens, table.size(1), first);
        at::Tensor out;
        if (args[2] == Py_None) {
            out = at::empty(shape, table.options().requires_grad(false));
        } else {
            out = tensor(args[2], "bad output tensor");
            require(out.sizes() == c10::IntArrayRef(shape) && out.scalar_type() == table.scalar_type() && out.device() == table.device() && out.is_contiguous(),
                    "bad output tensor");
        }
        return result(embed(table.data_ptr(), tokens.data_ptr(), out.data_ptr(), table.size(0), (int)table.size(1), s.count, s.words,
                            type_of(table.scalar_type()), (float)PyFloat_AS_DOUBLE(args[4]), s.flags, PyLong_AsVoidPtr(args[5])),
                      out, args[2] != Py_None);
    });
}

// backward(table, grad, tokens, out or None, channels_first, accumulate, scale, padding, stream)
PyObject* py_embed_backward(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        require(embed_backward, "not bound");
        require(count == 9 && PyFloat_Check(args[6]) && PyLong_Check(args[7]) && PyLong_Check(args[8]), "bad arguments");
        const at::Tensor& table = tensor(args[0], "table must be a tensor");
        const at::Tensor& grad = tensor(args[1], "grad must be a tensor");
        const at::Tensor& tokens = tensor(args[2], "tokens must be a tensor");
        const bool first = is_true(args[4]), accumulate = is_true(args[5]);
        require_table(table);
        const Sentences s = sentences_of(tokens, table, first);
        const auto shape = vectors_of(tokens, table.size(1), first);
        const int g = type_of(grad.scalar_type());
        require(grad.sizes() == c10::IntArrayRef(shape) && g >= 0 && grad.is_contiguous() && grad.device() == table.device(),
                "grad must be a contiguous tensor of the shape that forward gives");
        at::Tensor out;
        if (args[3] == Py_None) {
            require(!accumulate, "accumulate needs the tensor to add to");
            out = at::empty(table.sizes(), table.options().requires_grad(false));
        } else {
            out = tensor(args[3], "bad output tensor");
            require(out.sizes() == table.sizes() && out.device() == table.device() && out.is_contiguous(), "bad output tensor");
        }
        require(out.scalar_type() == at::kFloat || out.scalar_type() == grad.scalar_type(), "the table's gradient is fp32 or of the type of grad");
        const unsigned flags = s.flags | (accumulate ? SC_EMBED_ACCUMULATE : 0u);
        long long bytes = 0;
        int rc = embed_backward_workspace(table.size(0), (int)table.size(1), s.count, s.words, g, flags, &bytes);
        const c10::DataPtr work = rc == SC_OK ? workspace(bytes) : c10::DataPtr();
        if (rc == SC_OK)
            rc = embed_backward(grad.data_ptr(), tokens.data_ptr(), out.data_ptr(), table.size(0), (int)table.size(1), s.count, s.words, g,
                                type_of(out.scalar_type()), (float)PyFloat_AS_DOUBLE(args[6]), PyLong_AsLongLong(args[7]), flags,
                                work.get(), bytes, PyLong_AsVoidPtr(args[8]));
        return result(rc, out, args[3] != Py_None);
    });
}

// linear(x, scale of x or None, weight, scale, bias or None, K, relu, out or None, dtype or None, stream)
PyObject* py_linear(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        require(int8_linear, "not bound");
        require(count == 10 && PyLong_Check(args[5]) && PyLong_Check(args[9]), "bad arguments");
        const at::Tensor& x = tensor(args[0], "x must be a tensor");
        const at::Tensor& weight = tensor(args[2], "weight must be a tensor");
        const at::Tensor& w_scale = tensor(args[3], "scale must be a tensor");
        require(weight.scalar_type() == at::kChar && weight.dim() == 2 && w_scale.scalar_type() == at::kFloat, "weights must be 8-bit integers with fp32 scales");
        require(args[4] == Py_None || (THPVariable_Check(args[4]) && THPVariable_Unpack(args[4]).scalar_type() == at::kFloat), "bias must be fp32");
        const int64_t K = PyLong_AsLongLong(args[5]), N = weight.size(0), pitch = weight.size(1);
        require(K > 0, "K must be positive");
        const bool given = args[1] != Py_None;
        int64_t M = 0, ldx = 0;
        const float* x_scale = nullptr;
        int in = SC_I8;
        c10::SmallVector<int64_t, 5> shape;
        if (given) {
            const at::Tensor& scale = tensor(args[1], "scale must be a tensor");
            require(x.scalar_type() == at::kChar && x.dim() == 2 && x.size(1) == pitch && x.is_contiguous() && x.device() == weight.device() &&
                        scale.scalar_type() == at::kFloat && scale.dim() == 1 && scale.size(0) == x.size(0) && scale.is_contiguous() && scale.device() == x.device(),
                    "q must be [M][int8_pitch(K)] 8-bit integers and scale fp32 [M], as quantize makes them");
            M = x.size(0);
            ldx = pitch;
            x_scale = scale.data_ptr<float>();
            shape = {M, N};
        } else {
            in = type_of(x.scalar_type());
            require(in >= 0 && x.device() == weight.device() && x.dim() >= 1 && x.size(-1) == K,
                    "x must be a tensor [..., K] of fp32, binary16 or bfloat16 on the layer's device");
            M = x.numel() / K;
            if (x.is_contiguous()) {
                ldx = K;
            } else {
                require(x.dim() == 2 && (x.stride(1) == 1 || K == 1) && x.stride(0) >= K, "x must be contiguous, or [M][K] with contiguous rows that do not overlap");
                ldx = x.stride(0);
            }
            shape.assign(x.sizes().begin(), x.sizes().end());
            shape.back() = N;
        }
        require(M < (1ll << 31) && K < (1ll << 31) && N < (1ll << 31), "sizes past 32 bits");
        at::Tensor out;
        int64_t ldo = N;
        if (args[7] == Py_None) {
            at::ScalarType t = given ? at::kFloat : x.scalar_type();
            if (args[8] != Py_None) {
                require(THPDtype_Check(args[8]), "dtype must be a torch.dtype");
                t = reinterpret_cast<THPDtype*>(args[8])->scalar_type;
            }
            require(type_of(t) >= 0, "the output is fp32, binary16 or bfloat16");
            out = at::empty(shape, weight.options().dtype(t));
        } else {
            out = tensor(args[7], "bad output tensor");
            require(out.sizes() == c10::IntArrayRef(shape) && type_of(out.scalar_type()) >= 0 && out.device() == weight.device(), "bad output tensor");
            if (!out.is_contiguous()) {
                require(out.dim() == 2 && (out.stride(1) == 1 || N == 1) && out.stride(0) >= N, "bad output tensor");
                ldo = out.stride(0);
            }
        }
        const int o = type_of(out.scalar_type());
        long long bytes = 0;
        int rc = int8_linear_workspace((int)M, (int)N, (int)K, in, o, &bytes);
        const c10::DataPtr work = rc == SC_OK ? workspace(bytes) : c10::DataPtr();
        if (rc == SC_OK)
            rc = int8_linear(x.data_ptr(), x_scale, static_cast<const signed char*>(weight.data_ptr()), w_scale.data_ptr<float>(),
                             args[4] == Py_None ? nullptr : THPVariable_Unpack(args[4]).data_ptr<float>(), out.data_ptr(), (int)M, (int)N, (int)K, ldx, ldo,
                             in, o, is_true(args[6]) ? SC_EPILOGUE_RELU : 0u, work.get(), bytes, PyLong_AsVoidPtr(args[9]));
        return result(rc, out, args[7] != Py_None);
    });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<bind>("bind"), method<py_embed>("embed"), method<py_embed_backward>("embed_backward"), method<py_linear>("linear"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_text_torch", "Calls of the text model's operators on PyTorch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__text_torch() { return PyModule_Create(&module); }
