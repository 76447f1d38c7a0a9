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
decltype(&sparse_conv_linear_workspace) linear_workspace = nullptr;
decltype(&sparse_conv_linear) linear = nullptr;
decltype(&sparse_conv_linear_backward_workspace) linear_backward_workspace = nullptr;
decltype(&sparse_conv_linear_backward) linear_backward = nullptr;
decltype(&sparse_conv_cross_entropy) cross_entropy = nullptr;
decltype(&sparse_conv_adamw) adamw = nullptr;
decltype(&sparse_conv_adamw_count) adamw_count = nullptr;

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

// bind(...): addresses of the library's functions, in the order above.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    constexpr int kFunctions = 12;
    if (count != kFunctions || !all_numbers(args, 0, kFunctions)) {
        PyErr_SetString(PyExc_TypeError, "twelve addresses");
        return nullptr;
    }
    void* p[kFunctions];
    for (int i = 0; i < kFunctions; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    int next = 0;
    auto set = [&](auto& function) { function = reinterpret_cast<std::decay_t<decltype(function)>>(p[next++]); };
    set(embed);
    set(embed_backward_workspace);
    set(embed_backward);
    set(int8_linear_workspace);
    set(int8_linear);
    set(linear_workspace);
    set(linear);
    set(linear_backward_workspace);
    set(linear_backward);
    set(cross_entropy);
    set(adamw);
    set(adamw_count);
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

// Rows [M][cols] of a tensor [..., cols]: elements from one to the next (contiguous, or two dimensions and contiguous rows that do not overlap).
int64_t rows_of(const at::Tensor& t, const char* what)
{
    const int64_t cols = t.size(-1);
    if (t.is_contiguous()) return cols;
    require(t.dim() == 2 && (t.stride(1) == 1 || cols == 1) && t.stride(0) >= cols, what);
    return t.size(0) > 1 ? t.stride(0) : cols;
}

// A layer's weights [N][K].
struct Weights {
    int64_t N, K, ld;
    int dtype;
};
Weights weights_of(const at::Tensor& w)
{
    const int dtype = type_of(w.scalar_type());
    require(w.is_cuda() && dtype >= 0 && w.dim() == 2 && w.size(0) > 0 && w.size(1) > 0, "weight must be a CUDA tensor [N][K] of fp32, binary16 or bfloat16");
    const Weights r{w.size(0), w.size(1), rows_of(w, "the rows of weight must be contiguous"), dtype};
    require(r.N < (1ll << 31) && r.K < (1ll << 31), "sizes past 32 bits");
    return r;
}

// [..., N] where the input is [..., K].
c10::SmallVector<int64_t, 5> with_last(const at::Tensor& t, int64_t last)
{
    c10::SmallVector<int64_t, 5> shape(t.sizes().begin(), t.sizes().end());
    shape.back() = last;
    return shape;
}

void written(const at::Tensor& t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// What is not given in `o` (None) is made.
at::Tensor output(PyObject* o, c10::IntArrayRef shape, const at::TensorOptions& options, bool& given)
{
    given = THPVariable_Check(o);
    if (!given) return at::empty(shape, options);
    const at::Tensor& t = THPVariable_Unpack(o);
    require(t.sizes() == shape && t.scalar_type() == c10::typeMetaToScalarType(options.dtype()) && t.device() == options.device(), "bad output tensor");
    return t;
}

// layer(x, weight, bias or None, residual or None, out or None, keep, activation, stream): the output, or (output, what went into the activation)
PyObject* py_layer(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        require(linear, "not bound");
        require(count == 8 && PyLong_Check(args[6]) && PyLong_Check(args[7]), "bad arguments");
        const at::Tensor& x = tensor(args[0], "x must be a tensor");
        const at::Tensor& weight = tensor(args[1], "weight must be a tensor");
        const Weights w = weights_of(weight);
        require(x.scalar_type() == weight.scalar_type() && x.device() == weight.device() && x.dim() >= 1 && x.size(-1) == w.K,
                "x must be a tensor [..., K] of the weight's type and device");
        const int64_t M = x.numel() / w.K, ldx = rows_of(x, "x must be contiguous, or [M][K] with contiguous rows that do not overlap");
        require(M < (1ll << 31), "sizes past 32 bits");
        const float* bias = nullptr;
        if (args[2] != Py_None) {
            const at::Tensor& b = tensor(args[2], "bias must be a tensor");
            require(b.scalar_type() == at::kFloat && b.dim() == 1 && b.size(0) == w.N && b.is_contiguous() && b.device() == weight.device(), "bias must be an fp32 tensor [N]");
            bias = b.data_ptr<float>();
        }
        const auto shape = with_last(x, w.N);
        const void* residual = nullptr;
        int64_t ldr = w.N;
        if (args[3] != Py_None) {
            const at::Tensor& r = tensor(args[3], "residual must be a tensor");
            require(r.sizes() == c10::IntArrayRef(shape) && r.scalar_type() == x.scalar_type() && r.device() == x.device(), "residual must be a tensor of the output's shape, type and device");
            ldr = rows_of(r, "residual must be contiguous, or [M][N] with contiguous rows that do not overlap");
            residual = r.data_ptr();
        }
        const at::TensorOptions options = weight.options().requires_grad(false);
        bool given;
        const at::Tensor out = output(args[4], shape, options, given);
        const int64_t ldo = rows_of(out, "bad output tensor");
        const bool keep = is_true(args[5]);
        at::Tensor z;
        if (keep) z = at::empty(shape, options);
        long long bytes = 0;
        int rc = linear_workspace(x.data_ptr(), weight.data_ptr(), (int)M, (int)w.N, (int)w.K, ldx, w.ld, w.dtype, &bytes);
        const c10::DataPtr work = rc == SC_OK ? workspace(bytes) : c10::DataPtr();
        if (rc == SC_OK)
            rc = linear(x.data_ptr(), weight.data_ptr(), bias, residual, out.data_ptr(), keep ? z.data_ptr() : nullptr, (int)M, (int)w.N, (int)w.K, ldx, w.ld, ldr, ldo,
                        w.dtype, (int)PyLong_AsLong(args[6]), work.get(), bytes, PyLong_AsVoidPtr(args[7]));
        PyObject* first = result(rc, out, given);
        if (rc != SC_OK || !keep || !first) return first;
        PyObject* second = THPVariable_Wrap(z);
        PyObject* both = second ? PyTuple_Pack(2, first, second) : nullptr;
        Py_DECREF(first);
        Py_XDECREF(second);
        return both;
    });
}

// layer_backward(grad, x or None, weight, z or None, grad of x, of weight, of bias, accumulate, activation, stream): a tuple of the three
// gradients.  Each is False or None (not wanted: None comes back), True (made) or the tensor to write to.
PyObject* py_layer_backward(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        require(linear_backward, "not bound");
        require(count == 10 && PyLong_Check(args[8]) && PyLong_Check(args[9]), "bad arguments");
        const at::Tensor& grad = tensor(args[0], "grad must be a tensor");
        const at::Tensor& weight = tensor(args[2], "weight must be a tensor");
        const Weights w = weights_of(weight);
        const int act = (int)PyLong_AsLong(args[8]);
        const bool accumulate = is_true(args[7]);
        require(grad.scalar_type() == weight.scalar_type() && grad.device() == weight.device() && grad.dim() >= 1 && grad.size(-1) == w.N,
                "grad must be a tensor [..., N] of the weight's type and device");
        const int64_t M = grad.numel() / w.N, ldg = rows_of(grad, "grad must be contiguous, or [M][N] with contiguous rows that do not overlap");
        require(M < (1ll << 31), "sizes past 32 bits");
        const at::TensorOptions options = weight.options().requires_grad(false);
        const auto shape = with_last(grad, w.K);
        at::Tensor out[3];
        bool given[3] = {false, false, false};
        for (int i = 0; i < 3; ++i) {
            PyObject* o = args[4 + i];
            if (o == Py_None || o == Py_False) continue;
            require(o == Py_True || THPVariable_Check(o), "a gradient is True, False or the tensor to write to");
            require(i == 0 || !accumulate || o != Py_True, "accumulate needs the tensors to add to");
            if (i == 0) out[i] = output(o, shape, options, given[i]);
            else if (i == 1) out[i] = output(o, {w.N, w.K}, options, given[i]);
            else out[i] = output(o, {w.N}, options.dtype(at::kFloat), given[i]);
            require(out[i].is_contiguous(), "bad output tensor");
        }
        const void *x = nullptr, *z = nullptr;
        int64_t ldx = w.K;
        if (out[1].defined()) {
            const at::Tensor& t = tensor(args[1], "the gradient of the weight needs x");
            require(t.scalar_type() == weight.scalar_type() && t.device() == weight.device() && t.sizes() == c10::IntArrayRef(shape), "x must be a tensor [..., K] of the weight's type and device");
            ldx = rows_of(t, "x must be contiguous, or [M][K] with contiguous rows that do not overlap");
            x = t.data_ptr();
        }
        if (act != SC_ACT_NONE) {
            const at::Tensor& t = tensor(args[3], "an activation's gradient needs z, what went into it");
            require(t.scalar_type() == weight.scalar_type() && t.device() == weight.device() && t.sizes() == grad.sizes() && t.is_contiguous(), "z must be a contiguous tensor like grad");
            z = t.data_ptr();
        }
        void* p[3];
        for (int i = 0; i < 3; ++i) p[i] = out[i].defined() ? out[i].data_ptr() : nullptr;
        long long bytes = 0;
        int rc = linear_backward_workspace(grad.data_ptr(), x, weight.data_ptr(), p[0], p[1], p[2], (int)M, (int)w.N, (int)w.K, ldg, ldx, w.ld, w.dtype, act, &bytes);
        const c10::DataPtr work = rc == SC_OK ? workspace(bytes) : c10::DataPtr();
        if (rc == SC_OK)
            rc = linear_backward(grad.data_ptr(), z, x, weight.data_ptr(), p[0], p[1], static_cast<float*>(p[2]), (int)M, (int)w.N, (int)w.K, ldg, ldx, w.ld, w.dtype, act,
                                 accumulate ? SC_LINEAR_ACCUMULATE : 0u, work.get(), bytes, PyLong_AsVoidPtr(args[9]));
        for (int i = 0; i < 3; ++i)
            if (given[i]) written(out[i]);
        if (rc != SC_OK) return PyLong_FromLong(rc);
        PyObject* all = PyTuple_New(3);
        if (!all) return nullptr;
        for (int i = 0; i < 3; ++i) {
            PyObject* o = out[i].defined() ? THPVariable_Wrap(out[i]) : (Py_INCREF(Py_None), Py_None);
            if (!o) {
                Py_DECREF(all);
                return nullptr;
            }
            PyTuple_SET_ITEM(all, i, o);
        }
        return all;
    });
}

// cross_entropy(logits, labels, weights or None, grad, scale, stream): (losses, gradient of the logits or None); grad is False (none), True
// (made) or the tensor to write to.
PyObject* py_cross_entropy(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        require(cross_entropy, "not bound");
        require(count == 6 && PyFloat_Check(args[4]) && PyLong_Check(args[5]), "bad arguments");
        const at::Tensor& logits = tensor(args[0], "logits must be a tensor");
        const at::Tensor& labels = tensor(args[1], "labels must be a tensor");
        const int dtype = type_of(logits.scalar_type());
        require(logits.is_cuda() && dtype >= 0 && logits.dim() >= 1 && logits.size(-1) > 0, "logits must be a CUDA tensor [..., classes] of fp32, binary16 or bfloat16");
        const int64_t classes = logits.size(-1), rows = logits.numel() / classes, ldl = rows_of(logits, "logits must be contiguous, or [rows][classes] with contiguous rows that do not overlap");
        require(rows < (1ll << 31) && classes < (1ll << 31), "sizes past 32 bits");
        const c10::IntArrayRef outer = logits.sizes().slice(0, logits.dim() - 1);
        require((labels.scalar_type() == at::kLong || labels.scalar_type() == at::kInt) && labels.is_contiguous() && labels.device() == logits.device() && labels.sizes() == outer,
                "labels must be a contiguous tensor of 32- or 64-bit integers, one for each row of logits");
        const float* weights = nullptr;
        if (args[2] != Py_None) {
            const at::Tensor& t = tensor(args[2], "weights must be a tensor");
            require(t.scalar_type() == at::kFloat && t.is_contiguous() && t.device() == logits.device() && t.sizes() == outer, "weights must be a contiguous fp32 tensor, one for each row of logits");
            weights = t.data_ptr<float>();
        }
        const at::TensorOptions options = logits.options().requires_grad(false);
        const at::Tensor loss = at::empty(outer, options.dtype(at::kFloat));
        at::Tensor grad;
        bool given = false;
        int64_t ldg = classes;
        if (args[3] != Py_False && args[3] != Py_None) {
            require(args[3] == Py_True || THPVariable_Check(args[3]), "grad is True, False or the tensor to write to");
            grad = output(args[3], logits.sizes(), options, given);
            ldg = rows_of(grad, "bad output tensor");
        }
        const int rc = cross_entropy(logits.data_ptr(), labels.data_ptr(), weights, loss.data_ptr<float>(), grad.defined() ? grad.data_ptr() : nullptr, (int)rows, (int)classes,
                                     ldl, ldg, dtype, (float)PyFloat_AS_DOUBLE(args[4]), labels.scalar_type() == at::kLong ? SC_LOSS_LABELS_64 : 0u, PyLong_AsVoidPtr(args[5]));
        if (given) written(grad);
        if (rc != SC_OK) return PyLong_FromLong(rc);
        PyObject* first = THPVariable_Wrap(loss);
        PyObject* second = grad.defined() ? THPVariable_Wrap(grad) : (Py_INCREF(Py_None), Py_None);
        PyObject* both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
        Py_XDECREF(first);
        Py_XDECREF(second);
        return both;
    });
}

// adamw(params, grads, m, v, m_scale or None, v_scale or None, master or None, counted or None, (rate, beta1, beta2, eps, decay, scale), step, stream):
// a status.  params and grads are lists; a grad of None leaves its tensor alone.  States of all tensors lie in one array each, every tensor's at
// a whole number of blocks.  counted: (steps, memory for a step's number), then it is counted there.
PyObject* py_adamw(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        require(adamw && adamw_count, "not bound");
        require(count == 11 && PyList_Check(args[0]) && PyList_Check(args[1]) && PyTuple_Check(args[8]) && PyTuple_GET_SIZE(args[8]) == 6 && PyLong_Check(args[9]) && PyLong_Check(args[10]),
                "bad arguments");
        const Py_ssize_t tensors = PyList_GET_SIZE(args[0]);
        require(PyList_GET_SIZE(args[1]) == tensors, "a gradient for each parameter, or None");
        const at::Tensor& m = tensor(args[2], "m must be a tensor");
        const at::Tensor& v = tensor(args[3], "v must be a tensor");
        const bool small = m.scalar_type() == at::kFloat8_e4m3fn;
        const int64_t room = m.numel(), element = small ? 1 : 4;
        const int state_dtype = small ? (int)SC_E4M3 : (int)SC_F32;
        auto is_state = [&](const at::Tensor& t, at::ScalarType type, int64_t n) { return t.is_cuda() && t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.is_contiguous() && t.device() == m.device(); };
        const at::ScalarType type = small ? at::kFloat8_e4m3fn : at::kFloat;
        require(room % SC_ADAMW_BLOCK == 0 && is_state(m, type, room) && is_state(v, type, room), "states must be as the optimizer made them");
        float *m_scale = nullptr, *v_scale = nullptr, *master = nullptr;
        if (small) {
            const at::Tensor &a = tensor(args[4], "states of 8 bits need scales"), &b = tensor(args[5], "states of 8 bits need scales");
            require(is_state(a, at::kFloat, room / SC_ADAMW_BLOCK) && is_state(b, at::kFloat, room / SC_ADAMW_BLOCK), "states must be as the optimizer made them");
            m_scale = a.data_ptr<float>();
            v_scale = b.data_ptr<float>();
        }
        if (args[6] != Py_None) {
            const at::Tensor& t = tensor(args[6], "master must be a tensor");
            require(is_state(t, at::kFloat, room), "states must be as the optimizer made them");
            master = t.data_ptr<float>();
        }
        double rule[6];
        for (int i = 0; i < 6; ++i) rule[i] = PyFloat_AsDouble(PyTuple_GET_ITEM(args[8], i));
        if (PyErr_Occurred()) return nullptr;
        c10::SmallVector<sparse_conv_adamw_tensor, 64> list;
        list.reserve(tensors);
        int param_dtype = SC_F32, grad_dtype = SC_F32;
        int64_t at = 0;
        bool any = false;
        for (Py_ssize_t i = 0; i < tensors; ++i) {
            const at::Tensor& p = tensor(PyList_GET_ITEM(args[0], i), "parameters must be tensors");
            const int64_t n = p.numel(), begin = at;
            const int dtype = type_of(p.scalar_type());
            at += (n + SC_ADAMW_BLOCK - 1) / SC_ADAMW_BLOCK * SC_ADAMW_BLOCK;
            require(p.is_cuda() && p.device() == m.device() && dtype >= 0 && p.is_contiguous() && at <= room && (i == 0 || dtype == param_dtype),
                    "parameters must be contiguous CUDA tensors of one type and device, of the sizes that the optimizer was made for");
            param_dtype = dtype;
            PyObject* o = PyList_GET_ITEM(args[1], i);
            if (o == Py_None || n == 0) continue;
            const at::Tensor& g = tensor(o, "a gradient must be a tensor or None");
            const int gd = type_of(g.scalar_type());
            require(g.sizes() == p.sizes() && g.device() == p.device() && g.is_contiguous() && gd >= 0 && (!any || gd == grad_dtype),
                    "gradients must be contiguous tensors like their parameters, of one type");
            grad_dtype = gd;
            any = true;
            list.push_back({p.data_ptr(), g.data_ptr(), static_cast<char*>(m.data_ptr()) + begin * element, static_cast<char*>(v.data_ptr()) + begin * element,
                            small ? m_scale + begin / SC_ADAMW_BLOCK : nullptr, small ? v_scale + begin / SC_ADAMW_BLOCK : nullptr, master ? master + begin : nullptr, n});
        }
        require(at == room, "the parameters are not those that the optimizer was made for");
        void* stream = PyLong_AsVoidPtr(args[10]);
        const void* counted = nullptr;
        if (args[7] != Py_None) {
            require(PyTuple_Check(args[7]) && PyTuple_GET_SIZE(args[7]) == 2, "bad arguments");
            const at::Tensor &steps = tensor(PyTuple_GET_ITEM(args[7], 0), "steps must be a tensor"), &room_of = tensor(PyTuple_GET_ITEM(args[7], 1), "bad arguments");
            require(steps.scalar_type() == at::kLong && steps.numel() == 1 && steps.device() == m.device() && room_of.is_contiguous() && room_of.device() == m.device() &&
                        room_of.numel() * room_of.element_size() >= SC_ADAMW_COUNTED_BYTES, "bad arguments");
            counted = room_of.data_ptr();
            // (What the step would refuse must not count: its rule and types, then its arrays.)
            int rc = adamw(nullptr, 0, param_dtype, grad_dtype, state_dtype, rule[0], rule[1], rule[2], rule[3], rule[4], rule[5], 1, counted, stream);
            const int bytes_of[3] = {4, 2, 2};      // SC_F32, SC_F16, SC_BF16
            for (const sparse_conv_adamw_tensor& t : list) {
                const char *p = static_cast<const char*>(t.param), *g = static_cast<const char*>(t.grad);
                const int64_t p_bytes = t.count * bytes_of[param_dtype], g_bytes = t.count * bytes_of[grad_dtype];
                bool overlap = p < g + g_bytes && g < p + p_bytes;
                for (int i = 2; i < 7; ++i) {
                    if (args[i] == Py_None) continue;
                    const at::Tensor& state = THPVariable_Unpack(args[i]);
                    const char* from = static_cast<const char*>(state.data_ptr());
                    const char* end = from + state.numel() * state.element_size();
                    overlap = overlap || (p < end && from < p + p_bytes) || (g < end && from < g + g_bytes);
                }
                if (overlap) rc = SC_EINVAL;
            }
            if (rc != SC_OK) return PyLong_FromLong(rc);
            rc = adamw_count(static_cast<long long*>(steps.data_ptr()), room_of.data_ptr(), rule[1], rule[2], stream);
            if (rc != SC_OK) return PyLong_FromLong(rc);
            written(steps);
        }
        const int rc = adamw(list.data(), (int)list.size(), param_dtype, grad_dtype, state_dtype, rule[0], rule[1], rule[2], rule[3], rule[4], rule[5],
                             PyLong_AsLongLong(args[9]), counted, stream);
        for (Py_ssize_t i = 0; i < tensors; ++i)
            if (PyList_GET_ITEM(args[1], i) != Py_None) written(THPVariable_Unpack(PyList_GET_ITEM(args[0], i)));
        for (int i = 2; i < 7; ++i)
            if (args[i] != Py_None) written(THPVariable_Unpack(args[i]));
        return PyLong_FromLong(rc);
    });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<bind>("bind"), method<py_embed>("embed"), method<py_embed_backward>("embed_backward"), method<py_linear>("linear"),
                         method<py_layer>("layer"), method<py_layer_backward>("layer_backward"), method<py_cross_entropy>("cross_entropy"), method<py_adamw>("adamw"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_text_torch", "Calls of the text model's operators on PyTorch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__text_torch() { return PyModule_Create(&module); }
