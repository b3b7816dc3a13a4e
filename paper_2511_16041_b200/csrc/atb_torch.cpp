// The tensor side of the Python binding of layer norm, the gated feed-forward block and the linear cross entropy: checks,
// outputs, workspaces and the call of the C entry point, in one step.  Those calls come many times per layer and, for
// small sizes, take less time on the GPU than their marshalling does in Python (16 us for a layer norm against 6 here).
// The entry points of libatb.so are handed in by address (bind), so that this module serves whichever build of the
// library the package has loaded.  A function returns a tuple of tensors, or the status of an entry that refused the call;
// what the checks refuse here is a ValueError.  No C++ exception leaves a function.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <optional>
#include <vector>

#include "atb.h"

namespace {

#define ATB_ENTRIES(X)                                                                                                  \
    X(atb_layer_norm) X(atb_layer_norm_bfp16) X(atb_layer_norm_backward) X(atb_layer_norm_backward_workspace_bytes)     \
    X(atb_gated_ffn) X(atb_gated_ffn_workspace_bytes) X(atb_gated_ffn_backward) X(atb_gated_ffn_backward_workspace_bytes) \
    X(atb_linear_cross_entropy) X(atb_linear_cross_entropy_workspace_bytes) X(atb_linear_cross_entropy_backward)        \
    X(atb_linear_cross_entropy_backward_workspace_bytes) X(atb_bfp16_exp_bytes)
struct Entries {
#define ATB_ENTRY(name) decltype(&::name) name = nullptr;
    ATB_ENTRIES(ATB_ENTRY)
#undef ATB_ENTRY
};
Entries g_entry;

[[noreturn]] void refuse(const std::string& what) {
    PyErr_SetString(PyExc_ValueError, what.c_str());
    throw python_error();
}

// ---------------------------------------------------------------------------------- arguments
// The tensor behind an argument; None is an undefined tensor.
at::Tensor tensor(PyObject* o, const char* name) {
    if (o == Py_None) return {};
    if (!THPVariable_Check(o)) refuse(c10::str(name, ": a tensor"));
    return THPVariable_Unpack(o);
}
std::string told(const at::Tensor& t) {
    return t.defined() ? c10::str(t.sizes(), " of ", t.scalar_type(), " on ", t.device(), ", strides ", t.strides()) : std::string("None");
}
// A gradient: the tensor to write it to, None for a new one, False where it is not wanted.
struct Gradient {
    at::Tensor t;
    bool wanted;
    Gradient(PyObject* o, const char* name) : wanted(o != Py_False) {
        if (wanted) t = tensor(o, name);
    }
};
// The rest of a call: the device of its first matrix, which has to be the current one, its stream, and what it allocates.
// What a call allocates belongs to the stream that its kernels run on: a block that was freed on another stream may still
// be read or written there.
struct Call {
    c10::DeviceIndex device = -1;
    cudaStream_t stream = nullptr;
    std::optional<c10::cuda::CUDAStream> current;
    bool other_stream = false;             // not the current one
    std::vector<at::Tensor> made;          // results that were allocated on it

    Call(const at::Tensor& first, const char* name, PyObject* stream_arg) {
        if (!first.defined() || !first.is_cuda() || first.dim() != 2) refuse(c10::str(name, ": a CUDA matrix, got ", told(first)));
        device = first.get_device();
        if (device != c10::cuda::current_device()) refuse(c10::str(name, " is on cuda:", int(device), ", the current device is cuda:", int(c10::cuda::current_device())));
        current = c10::cuda::getCurrentCUDAStream(device);
        stream = current->stream();
        if (stream_arg != Py_None) {
            stream = static_cast<cudaStream_t>(PyLong_AsVoidPtr(stream_arg));
            if (PyErr_Occurred()) throw python_error();
            other_stream = stream != current->stream();
        }
    }
    // Row-major matrix on this device; returns its leading dimension (of a single row, whose stride says nothing, the columns).
    int64_t matrix(const at::Tensor& t, int64_t rows, int64_t cols, at::ScalarType type, const char* name) const {
        if (t.defined() && t.is_cuda() && t.get_device() == device && t.scalar_type() == type && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols &&
            (cols <= 1 || t.stride(1) == 1))
            return rows > 1 ? t.stride(0) : cols;
        refuse(c10::str(name, ": a row-major matrix [", rows, ", ", cols, "] of ", type, " on cuda:", int(device), ", got ", told(t)));
    }
    void vector(const at::Tensor& t, int64_t n, at::ScalarType type, const char* name) const {
        if (!(t.defined() && t.is_cuda() && t.get_device() == device && t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.is_contiguous()))
            refuse(c10::str(name, ": a contiguous vector of ", n, " ", type, " on cuda:", int(device), ", got ", told(t)));
    }
    at::Tensor make(at::IntArrayRef size, at::ScalarType type) const {
        const auto options = at::TensorOptions().dtype(type).device(c10::Device(c10::kCUDA, device));
        if (!other_stream) return at::empty(size, options);
        // 0 and 1 are names of the default stream
        const bool is_default = reinterpret_cast<uintptr_t>(stream) <= 1;
        const c10::cuda::CUDAStreamGuard guard(is_default ? c10::cuda::getDefaultCUDAStream(device) : c10::cuda::getStreamFromExternal(stream, device));
        return at::empty(size, options);
    }
    at::Tensor make_result(at::IntArrayRef size, at::ScalarType type) {
        at::Tensor t = make(size, type);
        if (other_stream) made.push_back(t);
        return t;
    }
    // An output: the caller's, checked, or a new one.
    int64_t out_matrix(at::Tensor& t, int64_t rows, int64_t cols, at::ScalarType type, const char* name) {
        if (t.defined()) return matrix(t, rows, cols, type, name);
        t = make_result({rows, cols}, type);
        return cols;
    }
    int64_t out_matrix(Gradient& g, int64_t rows, int64_t cols, at::ScalarType type, const char* name) {
        return g.wanted ? out_matrix(g.t, rows, cols, type, name) : cols;
    }
    void out_vector(Gradient& g, int64_t n, at::ScalarType type, const char* name) {
        if (g.wanted) out_vector(g.t, n, type, name);
    }
    void out_vector(at::Tensor& t, int64_t n, at::ScalarType type, const char* name) {
        if (t.defined()) vector(t, n, type, name);
        else t = make_result({n}, type);
    }
    void out_contiguous(at::Tensor& t, int64_t rows, int64_t cols, at::ScalarType type, const char* name) {
        if (out_matrix(t, rows, cols, type, name) != cols) refuse(c10::str(name, ": contiguous"));
    }
    // Room for `need` bytes: the caller's workspace, or a new one.
    size_t workspace(at::Tensor& t, size_t need) const {
        if (!t.defined()) {
            if (need == 0) return 0;
            t = make({static_cast<int64_t>(need)}, at::kByte);
            return need;
        }
        if (!t.is_cuda() || t.get_device() != device || !t.is_contiguous()) refuse("workspace: contiguous, on the tensors' device");
        return t.nbytes();
    }
    // Ends the call.  The caller will use the results on the current stream (once it has waited for the one given): they are not
    // handed out again before that is through with them either.
    PyObject* done(atb_status_t status, std::initializer_list<at::Tensor> result) {
        for (const at::Tensor& t : made) t.record_stream(*current);
        if (status != ATB_OK) return PyLong_FromLong(status);
        PyObject* tuple = PyTuple_New(static_cast<Py_ssize_t>(result.size()));
        if (!tuple) throw python_error();
        Py_ssize_t i = 0;
        for (const at::Tensor& t : result) PyTuple_SET_ITEM(tuple, i++, THPVariable_Wrap(t));
        return tuple;
    }
};

int type_code(at::ScalarType type, const char* name) {
    if (type == at::kFloat) return ATB_F32;
    if (type == at::kBFloat16) return ATB_BF16;
    refuse(c10::str(name, ": float32 or bfloat16, got ", type));
}
int type_code(const at::Tensor& t, const char* name) { return type_code(t.scalar_type(), name); }
void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float* fptr(const at::Tensor& t) { return static_cast<float*>(ptr(t)); }
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
// The number of an activation; what is none, an int's excess or a flag of the entries, becomes -1, which they refuse.
int activation(PyObject* o) {
    const int64_t v = integer(o);
    return v >= 0 && v < ATB_KEEP_F32 ? static_cast<int>(v) : -1;
}
int with_kept(int act, at::ScalarType kept) { return act >= 0 && kept == at::kFloat ? act | ATB_KEEP_F32 : act; }
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v == 1;
}
void expect(Py_ssize_t given, Py_ssize_t wanted) {
    if (given != wanted) refuse(c10::str("takes ", wanted, " arguments, got ", given));
}

// ---------------------------------------------------------------------------------- layer norm
// Type code of the weights; of either where only one is given.
int norm_weights(const Call& c, const at::Tensor& W, const at::Tensor& B, int64_t N) {
    const at::Tensor& given = W.defined() ? W : B;
    if (!given.defined()) return ATB_F32;
    if (W.defined()) c.vector(W, N, given.scalar_type(), "W");
    if (B.defined()) c.vector(B, N, given.scalar_type(), "B");
    return type_code(given, W.defined() ? "W" : "B");
}

// (X, W, B, eps, Y, mean, rstd, stream) -> (Y, mean, rstd)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 8);
    const at::Tensor X = tensor(a[0], "X"), W = tensor(a[1], "W"), B = tensor(a[2], "B");
    at::Tensor Y = tensor(a[4], "Y"), mean = tensor(a[5], "mean"), rstd = tensor(a[6], "rstd");
    const double eps = PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) throw python_error();
    Call c(X, "X", a[7]);
    const int64_t M = X.size(0), N = X.size(1);
    const int x_type = type_code(X, "X");
    const int64_t ldx = c.matrix(X, M, N, X.scalar_type(), "X");
    const int w_type = norm_weights(c, W, B, N);
    const int64_t ldy = c.out_matrix(Y, M, N, X.scalar_type(), "Y");
    c.out_vector(mean, M, at::kFloat, "mean");
    c.out_vector(rstd, M, at::kFloat, "rstd");
    return c.done(g_entry.atb_layer_norm(M, N, x_type, ptr(X), ldx, w_type, ptr(W), ptr(B), static_cast<float>(eps), ptr(Y), ldy, fptr(mean), fptr(rstd),
                                         c.stream), {Y, mean, rstd});
    END_HANDLE_TH_ERRORS
}

// (X, W, B, eps, mant, exp, mean, rstd, stream) -> (mant, exp, mean, rstd)
PyObject* layer_norm_bfp16(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 9);
    const at::Tensor X = tensor(a[0], "X"), W = tensor(a[1], "W"), B = tensor(a[2], "B");
    at::Tensor mant = tensor(a[4], "mant"), exp = tensor(a[5], "exp"), mean = tensor(a[6], "mean"), rstd = tensor(a[7], "rstd");
    const double eps = PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) throw python_error();
    Call c(X, "X", a[8]);
    const int64_t M = X.size(0), N = X.size(1);
    const int x_type = type_code(X, "X");
    const int64_t ldx = c.matrix(X, M, N, X.scalar_type(), "X");
    const int w_type = norm_weights(c, W, B, N);
    c.out_contiguous(mant, M, N, at::kChar, "mant");
    c.out_vector(exp, static_cast<int64_t>(g_entry.atb_bfp16_exp_bytes(M, N)), at::kByte, "exp");
    c.out_vector(mean, M, at::kFloat, "mean");
    c.out_vector(rstd, M, at::kFloat, "rstd");
    return c.done(g_entry.atb_layer_norm_bfp16(M, N, x_type, ptr(X), ldx, w_type, ptr(W), ptr(B), static_cast<float>(eps), static_cast<int8_t*>(ptr(mant)),
                                               static_cast<uint8_t*>(ptr(exp)), fptr(mean), fptr(rstd), c.stream), {mant, exp, mean, rstd});
    END_HANDLE_TH_ERRORS
}

// (dY, X, W, mean, rstd, dX, dW, dB, workspace, stream) -> (dX, dW, dB)
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 10);
    const at::Tensor dY = tensor(a[0], "dY"), X = tensor(a[1], "X"), W = tensor(a[2], "W"), mean = tensor(a[3], "mean"), rstd = tensor(a[4], "rstd");
    Gradient dX(a[5], "dX"), dW(a[6], "dW"), dB(a[7], "dB");
    at::Tensor ws = tensor(a[8], "workspace");
    Call c(X, "X", a[9]);
    const int64_t M = X.size(0), N = X.size(1);
    const at::ScalarType type = X.scalar_type(), w_dtype = W.defined() ? W.scalar_type() : at::kFloat;
    const int x_type = type_code(X, "X");
    const int64_t ldx = c.matrix(X, M, N, type, "X"), lddy = c.matrix(dY, M, N, type, "dY");
    if (W.defined()) c.vector(W, N, w_dtype, "W");
    c.vector(mean, M, at::kFloat, "mean");
    c.vector(rstd, M, at::kFloat, "rstd");
    const int64_t lddx = c.out_matrix(dX, M, N, type, "dX");
    c.out_vector(dW, N, w_dtype, "dW");
    c.out_vector(dB, N, w_dtype, "dB");
    const size_t bytes = c.workspace(ws, dW.wanted || dB.wanted ? g_entry.atb_layer_norm_backward_workspace_bytes(M, N) : 0);
    return c.done(g_entry.atb_layer_norm_backward(M, N, x_type, ptr(dY), lddy, ptr(X), ldx, type_code(w_dtype, "W"), ptr(W), fptr(mean), fptr(rstd), ptr(dX.t), lddx,
                                                  ptr(dW.t), ptr(dB.t), ptr(ws), bytes, c.stream), {dX.t, dW.t, dB.t});
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------------- gated feed-forward block
struct FfnShapes {
    int64_t M, D, F, ldx, ldw, ldwd;
    FfnShapes(const Call& c, const at::Tensor& X, const at::Tensor& Wg, const at::Tensor& Wu, const at::Tensor& Wd) {
        if (!Wd.defined() || Wd.dim() != 2) refuse(c10::str("Wd: a matrix, got ", told(Wd)));
        M = X.size(0); D = X.size(1); F = Wd.size(0);
        ldx = c.matrix(X, M, D, at::kBFloat16, "X");
        ldw = c.matrix(Wg, D, F, at::kBFloat16, "Wg");
        ldwd = c.matrix(Wd, F, D, at::kBFloat16, "Wd");
        if (c.matrix(Wu, D, F, at::kBFloat16, "Wu") != ldw) refuse("Wg and Wu need the same row stride");
    }
};

// Type of G and U: of those given, which have to agree, else of `fallback`.
at::ScalarType kept_type(const at::Tensor& G, const at::Tensor& U, at::ScalarType fallback) {
    const at::ScalarType type = G.defined() ? G.scalar_type() : U.defined() ? U.scalar_type() : fallback;
    if (type != at::kFloat && type != at::kBFloat16) refuse(c10::str("G and U: float32 or bfloat16, got ", type));
    return type;
}

// (X, Wg, Wu, Wd, act, save, Y, H, G, U, workspace, stream) -> (Y, H, G, U), G and U None where not saved; save: a truth value, or the
// type of G and U
PyObject* gated_ffn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 12);
    const at::Tensor X = tensor(a[0], "X"), Wg = tensor(a[1], "Wg"), Wu = tensor(a[2], "Wu"), Wd = tensor(a[3], "Wd");
    const int act = activation(a[4]);
    at::Tensor Y = tensor(a[6], "Y"), H = tensor(a[7], "H"), G = tensor(a[8], "G"), U = tensor(a[9], "U"), ws = tensor(a[10], "workspace");
    const bool typed = THPDtype_Check(a[5]), save = typed || truth(a[5]) || G.defined() || U.defined();
    const at::ScalarType kept = kept_type(G, U, typed ? reinterpret_cast<THPDtype*>(a[5])->scalar_type : at::kFloat);
    Call c(X, "X", a[11]);
    const FfnShapes s(c, X, Wg, Wu, Wd);
    const int64_t ldy = c.out_matrix(Y, s.M, s.D, at::kBFloat16, "Y");
    c.out_contiguous(H, s.M, s.F, at::kBFloat16, "H");
    if (save) {
        c.out_contiguous(G, s.M, s.F, kept, "G");
        c.out_contiguous(U, s.M, s.F, kept, "U");
    }
    const size_t bytes = c.workspace(ws, g_entry.atb_gated_ffn_workspace_bytes(s.M, s.D, s.F));
    return c.done(g_entry.atb_gated_ffn(s.M, s.D, s.F, with_kept(act, kept), ptr(X), s.ldx, ptr(Wg), ptr(Wu), s.ldw, ptr(Wd), s.ldwd, ptr(Y), ldy, ptr(H), ptr(G), ptr(U),
                                        ptr(ws), bytes, c.stream), {Y, H, G, U});
    END_HANDLE_TH_ERRORS
}

// (dY, X, Wg, Wu, Wd, H, G, U, act, dX, dWg, dWu, dWd, workspace, stream) -> (dX, dWg, dWu, dWd)
PyObject* gated_ffn_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 15);
    const at::Tensor dY = tensor(a[0], "dY"), X = tensor(a[1], "X"), Wg = tensor(a[2], "Wg"), Wu = tensor(a[3], "Wu"), Wd = tensor(a[4], "Wd");
    const at::Tensor H = tensor(a[5], "H"), G = tensor(a[6], "G"), U = tensor(a[7], "U");
    const int act = activation(a[8]);
    Gradient dX(a[9], "dX"), dWg(a[10], "dWg"), dWu(a[11], "dWu"), dWd(a[12], "dWd");
    at::Tensor ws = tensor(a[13], "workspace");
    if (dWg.wanted != dWu.wanted) refuse("dWg and dWu: both or neither");
    Call c(X, "X", a[14]);
    const FfnShapes s(c, X, Wg, Wu, Wd);
    const at::ScalarType bf16 = at::kBFloat16;
    const int64_t lddy = c.matrix(dY, s.M, s.D, bf16, "dY");
    const at::ScalarType kept = kept_type(G, U, bf16);
    if (c.matrix(H, s.M, s.F, bf16, "H") != s.F || c.matrix(G, s.M, s.F, kept, "G") != s.F || c.matrix(U, s.M, s.F, kept, "U") != s.F)
        refuse("H, G, U: contiguous");
    const int64_t lddx = c.out_matrix(dX, s.M, s.D, bf16, "dX"), lddw = c.out_matrix(dWg, s.D, s.F, bf16, "dWg");
    if (c.out_matrix(dWu, s.D, s.F, bf16, "dWu") != lddw) refuse("dWg and dWu need the same row stride");
    const int64_t lddwd = c.out_matrix(dWd, s.F, s.D, bf16, "dWd");
    const size_t bytes = c.workspace(ws, g_entry.atb_gated_ffn_backward_workspace_bytes(s.M, s.D, s.F));
    return c.done(g_entry.atb_gated_ffn_backward(s.M, s.D, s.F, with_kept(act, kept), ptr(dY), lddy, ptr(X), s.ldx, ptr(Wg), ptr(Wu), s.ldw, ptr(Wd), s.ldwd, ptr(H), ptr(G),
                                                 ptr(U), ptr(dX.t), lddx, ptr(dWg.t), ptr(dWu.t), lddw, ptr(dWd.t), lddwd, ptr(ws), bytes, c.stream),
                  {dX.t, dWg.t, dWu.t, dWd.t});
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------------- linear cross entropy
struct HeadShapes {
    int64_t M, V, D, ldx, ldw;
    HeadShapes(const Call& c, const at::Tensor& X, const at::Tensor& W, const at::Tensor& labels) {
        if (!W.defined() || W.dim() != 2) refuse(c10::str("W: a matrix, got ", told(W)));
        M = X.size(0); D = X.size(1); V = W.size(0);
        ldx = c.matrix(X, M, D, at::kBFloat16, "X");
        ldw = c.matrix(W, V, D, at::kBFloat16, "W");
        c.vector(labels, M, at::kLong, "labels");
    }
};

// (X, W, labels, ignore_index, loss, lse, workspace, stream) -> (loss, lse)
PyObject* linear_cross_entropy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 8);
    const at::Tensor X = tensor(a[0], "X"), W = tensor(a[1], "W"), labels = tensor(a[2], "labels");
    const int64_t ignore = integer(a[3]);
    at::Tensor loss = tensor(a[4], "loss"), lse = tensor(a[5], "lse"), ws = tensor(a[6], "workspace");
    Call c(X, "X", a[7]);
    const HeadShapes s(c, X, W, labels);
    c.out_vector(loss, s.M, at::kFloat, "loss");
    c.out_vector(lse, s.M, at::kFloat, "lse");
    const size_t bytes = c.workspace(ws, g_entry.atb_linear_cross_entropy_workspace_bytes(s.M, s.V, s.D));
    return c.done(g_entry.atb_linear_cross_entropy(s.M, s.V, s.D, ptr(X), s.ldx, ptr(W), s.ldw, static_cast<const int64_t*>(ptr(labels)), ignore, fptr(loss),
                                                   fptr(lse), ptr(ws), bytes, c.stream), {loss, lse});
    END_HANDLE_TH_ERRORS
}

// (dloss, X, W, labels, lse, ignore_index, dX, dW, piece, workspace, stream) -> (dX, dW)
PyObject* linear_cross_entropy_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 11);
    const at::Tensor dloss = tensor(a[0], "dloss"), X = tensor(a[1], "X"), W = tensor(a[2], "W"), labels = tensor(a[3], "labels"), lse = tensor(a[4], "lse");
    const int64_t ignore = integer(a[5]), piece = integer(a[8]);
    Gradient dX(a[6], "dX"), dW(a[7], "dW");
    at::Tensor ws = tensor(a[9], "workspace");
    Call c(X, "X", a[10]);
    const HeadShapes s(c, X, W, labels);
    c.vector(dloss, s.M, at::kFloat, "dloss");
    c.vector(lse, s.M, at::kFloat, "lse");
    const int64_t lddx = c.out_matrix(dX, s.M, s.D, at::kBFloat16, "dX"), lddw = c.out_matrix(dW, s.V, s.D, at::kBFloat16, "dW");
    const size_t bytes = c.workspace(ws, g_entry.atb_linear_cross_entropy_backward_workspace_bytes(s.M, s.V, s.D, piece));
    return c.done(g_entry.atb_linear_cross_entropy_backward(s.M, s.V, s.D, ptr(X), s.ldx, ptr(W), s.ldw, static_cast<const int64_t*>(ptr(labels)), ignore,
                                                            fptr(lse), fptr(dloss), ptr(dX.t), lddx, ptr(dW.t), lddw, piece, ptr(ws), bytes, c.stream),
                  {dX.t, dW.t});
    END_HANDLE_TH_ERRORS
}

// (name, address) of an entry point of the library
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    expect(n, 2);
    const char* name = PyUnicode_AsUTF8(a[0]);
    void* address = name ? PyLong_AsVoidPtr(a[1]) : nullptr;
    if (PyErr_Occurred()) throw python_error();
#define ATB_ENTRY(entry) \
    if (std::strcmp(name, #entry) == 0) { g_entry.entry = reinterpret_cast<decltype(g_entry.entry)>(address); Py_RETURN_NONE; }
    ATB_ENTRIES(ATB_ENTRY)
#undef ATB_ENTRY
    refuse(c10::str("no entry point ", name));
    END_HANDLE_TH_ERRORS
}

#define ATB_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {ATB_METHOD(layer_norm), ATB_METHOD(layer_norm_bfp16), ATB_METHOD(layer_norm_backward), ATB_METHOD(gated_ffn),
                           ATB_METHOD(gated_ffn_backward), ATB_METHOD(linear_cross_entropy), ATB_METHOD(linear_cross_entropy_backward), ATB_METHOD(bind),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_atb_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__atb_torch() {
    PyObject* m = PyModule_Create(&g_module);
#define ATB_ENTRY(entry) #entry,
    static const char* const names[] = {ATB_ENTRIES(ATB_ENTRY)};
#undef ATB_ENTRY
    if (!m) return nullptr;
    PyObject* list = PyTuple_New(static_cast<Py_ssize_t>(sizeof names / sizeof names[0]));
    for (size_t i = 0; list && i < sizeof names / sizeof names[0]; ++i) PyTuple_SET_ITEM(list, static_cast<Py_ssize_t>(i), PyUnicode_FromString(names[i]));
    if (!list || PyModule_AddObject(m, "ENTRIES", list) < 0) return nullptr;
    return m;
}
