// Python entry points of the operators whose smallest calls are bound by the host: routing from logits, 8-bit products, 8-bit
// experts, the layer of a few tokens and the joins between blocks.  Same job as the ctypes binding (check the tensors, allocate the outputs, fill the argument struct, call the C
// entry point of libmok.so), in C++: through ctypes a call took 9 to 11 us of host time against 3 us of launch, because every
// allocation, attribute and struct field is an interpreted call.  Built as _binding.so beside libmok.so.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>

#include "mok.h"

namespace {

PyObject* g_error = nullptr;             // mok.MokError

// ------------------------------------------------------------------------------------------------- arguments of a call
// A string for a message (there are Python strings that have no UTF-8 form)
std::string text(PyObject* o) {
    const char* s = PyUnicode_AsUTF8(o);
    if (s) return s;
    PyErr_Clear();
    return "?";
}

// A function's argument names, interned: a caller's keywords mostly are the same objects.
template <int N>
struct Names {
    const char* const* text;
    PyObject* interned[N];
    explicit Names(const char* const (&names)[N]) : text(names) {
        for (int i = 0; i < N; ++i) interned[i] = PyUnicode_InternFromString(names[i]);
    }
};
// Positional and keyword arguments by name; `required` of them have to be there.
template <int N>
struct Call {
    PyObject* v[N] = {};
    Call(const char* function, const Names<N>& names, int required, PyObject* const* args, Py_ssize_t n_args, PyObject* kwnames) {
        if (n_args > N) throw_type(function, "too many positional arguments");
        for (Py_ssize_t i = 0; i < n_args; ++i) v[i] = args[i];
        const Py_ssize_t n_kw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
        int next = (int)n_args % N;
        for (Py_ssize_t q = 0; q < n_kw; ++q) {
            PyObject* name = PyTuple_GET_ITEM(kwnames, q);
            int at = -1;
            for (int i = 0; i < N && at < 0; ++i, next = next + 1 == N ? 0 : next + 1)   // (keywords mostly come in order)
                if (name == names.interned[next]) at = next;
            for (int i = 0; i < N && at < 0; ++i)
                if (PyUnicode_CompareWithASCIIString(name, names.text[i]) == 0) at = i;
            if (at < 0) throw_type(function, std::string("unexpected argument ") + text(name));
            if (v[at]) throw_type(function, std::string("argument given twice: ") + names.text[at]);
            v[at] = args[n_args + q];
        }
        for (int i = 0; i < N; ++i) {
            if (v[i] == Py_None) v[i] = nullptr;
            if (i < required && !v[i]) throw_type(function, std::string("missing argument ") + names.text[i]);
        }
    }
    static void throw_type(const char* function, const std::string& what) {
        TORCH_CHECK_TYPE(false, function, "(): ", what);
    }
};

const at::Tensor& tensor(const char* name, PyObject* o) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, ": expected a tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
int64_t integer(PyObject* o, int64_t otherwise) {
    if (!o) return otherwise;
    const long long r = PyLong_AsLongLong(o);
    if (r == -1 && PyErr_Occurred()) throw python_error();
    return r;
}
int32_t small(const char* name, PyObject* o, int64_t otherwise) {
    const int64_t r = integer(o, otherwise);
    TORCH_CHECK_VALUE(r >= INT32_MIN && r <= INT32_MAX, name, ": out of range: ", r);
    return (int32_t)r;
}
double number(PyObject* o, double otherwise) {
    if (!o) return otherwise;
    const double r = PyFloat_AsDouble(o);
    if (r == -1.0 && PyErr_Occurred()) throw python_error();
    return r;
}
bool truth(PyObject* o, bool otherwise) {
    if (!o) return otherwise;
    const int r = PyObject_IsTrue(o);
    if (r < 0) throw python_error();
    return r != 0;
}
int32_t score(PyObject* o) {
    if (!o) return MOK_SCORE_SOFTMAX;
    TORCH_CHECK_TYPE(PyUnicode_Check(o), "score: expected a string");
    if (PyUnicode_CompareWithASCIIString(o, "softmax") == 0) return MOK_SCORE_SOFTMAX;
    if (PyUnicode_CompareWithASCIIString(o, "sigmoid") == 0) return MOK_SCORE_SIGMOID;
    TORCH_CHECK_VALUE(false, "score: expected \"softmax\" or \"sigmoid\", got \"", text(o), "\"");
}
int32_t type_of(const char* name, at::ScalarType t) {
    if (t == at::kBFloat16) return MOK_TYPE_BF16;
    if (t == at::kHalf) return MOK_TYPE_F16;
    TORCH_CHECK_VALUE(t == at::kFloat, name, ": expected bfloat16, float16 or float32, got ", t);
    return MOK_TYPE_F32;
}
at::ScalarType dtype_of(PyObject* o, at::ScalarType otherwise) {
    if (!o) return otherwise;
    TORCH_CHECK_TYPE(THPDtype_Check(o), "out_dtype: expected a torch.dtype");
    return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

// A matrix [rows, >= width] whose last index is contiguous, on `device`; returns the elements between its rows.
int64_t rows(const char* name, const at::Tensor& t, int64_t width, c10::Device device) {
    TORCH_CHECK_VALUE(t.dim() == 2 && t.size(1) >= width && (t.size(1) <= 1 || t.stride(1) == 1) && t.device() == device, name,
                      ": expected rows of ", width, " contiguous elements on ", device, ", got shape ", t.sizes(), ", strides ",
                      t.strides(), " on ", t.device());
    return t.size(0) > 1 ? t.stride(0) : t.size(1);
}
// A contiguous tensor of that shape and type on `device`; returns its address.
void* packed(const char* name, const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type, c10::Device device) {
    TORCH_CHECK_VALUE(t.sizes() == shape && t.scalar_type() == type && t.device() == device && t.is_contiguous(), name,
                      ": expected a contiguous tensor ", shape, " of ", type, " on ", device, ", got shape ", t.sizes(), ", strides ",
                      t.strides(), ", ", t.scalar_type(), " on ", t.device());
    return t.data_ptr();
}
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, c10::Device device) {
    return at::Tensor(at::detail::empty_cuda(shape, type, device, std::nullopt));
}

// Device and stream of a call: the first tensor's device becomes current; with stream=, so does that stream, so that outputs and
// scratch belong to the stream that writes them.
struct Where {
    c10::Device device;
    c10::cuda::OptionalCUDAGuard device_guard;
    std::optional<c10::cuda::CUDAStreamGuard> stream_guard;
    void* stream;
    Where(const char* function, const at::Tensor& first, PyObject* stream_object) : device(first.device()), stream(nullptr) {
        TORCH_CHECK_VALUE(device.is_cuda(), function, ": tensors have to be on a CUDA device, got ", device);
        if (device.index() != c10::cuda::current_device()) device_guard.set_device(device);
        if (stream_object) {
            PyObject* raw = PyObject_GetAttrString(stream_object, "cuda_stream");
            if (!raw) throw python_error();
            const unsigned long long p = PyLong_AsUnsignedLongLong(raw);
            Py_DECREF(raw);
            if (PyErr_Occurred()) throw python_error();
            stream_guard.emplace(c10::cuda::getStreamFromExternal(reinterpret_cast<cudaStream_t>(p), device.index()));
            stream = reinterpret_cast<void*>(p);
        } else {
            stream = c10::cuda::getCurrentCUDAStream(device.index()).stream();
        }
    }
};

void check(int status) {
    if (status == MOK_OK) return;
    PyObject* e = PyObject_CallFunction(g_error ? g_error : PyExc_RuntimeError, "i", status);
    if (e) {
        PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e)), e);
        Py_DECREF(e);
    }
    throw python_error();
}

// 256-byte aligned scratch of `bytes`: the caller's tensor, or a new one (kept in `own` until the launches are enqueued)
void scratch(PyObject* given, size_t bytes, c10::Device device, at::Tensor& own, void** at, size_t* have) {
    if (given) {
        const at::Tensor& t = tensor("workspace", given);
        TORCH_CHECK_VALUE(t.is_contiguous() && t.device() == device, "workspace: expected a contiguous tensor on ", device);
        const uintptr_t p = reinterpret_cast<uintptr_t>(t.data_ptr()), a = (p + 255) & ~uintptr_t(255);
        const size_t n = t.nbytes();
        *at = reinterpret_cast<void*>(a);
        *have = n > a - p ? n - (a - p) : 0;
    } else if (bytes) {
        own = make({(int64_t)bytes}, at::kByte, device);
        *at = own.data_ptr();
        *have = bytes;
    }
}

struct Weights {                         // the tensors of an I8Weights
    at::Tensor codes, scales, max;
    Weights(const char* name, PyObject* o) {
        static PyObject *codes_name = PyUnicode_InternFromString("codes"), *scales_name = PyUnicode_InternFromString("scales"),
                        *max_name = PyUnicode_InternFromString("max");
        codes = get(name, o, codes_name);
        scales = get(name, o, scales_name);
        max = get(name, o, max_name);
    }
    static at::Tensor get(const char* name, PyObject* o, PyObject* attribute) {
        PyObject* v = PyObject_GetAttr(o, attribute);
        if (!v) throw python_error();
        at::Tensor t;
        if (v != Py_None) {
            if (!THPVariable_Check(v)) {
                Py_DECREF(v);
                TORCH_CHECK_TYPE(false, name, ": expected I8Weights");
            }
            t = THPVariable_Unpack(v);
        }
        Py_DECREF(v);
        return t;
    }
};

// -------------------------------------------------------------------------------------------------------- entry points
const char GATE_DOC[] =
    "mok_gate(logits, k, bias=None, score='softmax', n_groups=1, topk_groups=1, group_top=2, renormalise=True, scale=1.0, stream=None)\n"
    "--\n\n"
    "Routing from logits [T, E] (bf16, fp16 or fp32): returns (topk_idx int32 [T, k], topk_w fp32 [T, k]).  score: 'softmax' or\n"
    "'sigmoid'; bias fp32 [E] takes part in the selection only; see include/mok.h for groups and weights.  Outside of autograd,\n"
    "like the layer's own calls: logits that require a gradient get theirs from mok_gate_backward.";
PyObject* gate(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"logits", "k", "bias", "score", "n_groups", "topk_groups", "group_top", "renormalise", "scale", "stream"};
    static const Names<10> names(texts);
    const Call<10> c("mok_gate", names, 2, args, n, kw);
    const at::Tensor& logits = tensor("logits", c.v[0]);
    const Where w("mok_gate", logits, c.v[9]);
    mok_gate_args a = {};
    a.logits_stride = rows("logits", logits, 0, w.device);
    a.logits = logits.data_ptr();
    a.logits_type = type_of("logits", logits.scalar_type());
    a.T = (int32_t)logits.size(0);
    a.E = (int32_t)logits.size(1);
    a.k = small("k", c.v[1], 0);
    if (c.v[2]) a.bias = static_cast<const float*>(packed("bias", tensor("bias", c.v[2]), {logits.size(1)}, at::kFloat, w.device));
    a.score = score(c.v[3]);
    a.n_groups = small("n_groups", c.v[4], 1);
    a.topk_groups = small("topk_groups", c.v[5], 1);
    a.group_top = small("group_top", c.v[6], 2);
    a.renormalise = truth(c.v[7], true);
    a.scale = (float)number(c.v[8], 1.0);
    TORCH_CHECK_VALUE(logits.size(0) <= INT32_MAX && logits.size(1) <= INT32_MAX, "logits: too large");
    if (a.k < 1 || a.k > a.E) check(MOK_ERR_SHAPE);     // (before outputs of that size are allocated)
    at::Tensor idx = make({a.T, a.k}, at::kInt, w.device), weight = make({a.T, a.k}, at::kFloat, w.device);
    a.topk_idx = static_cast<int32_t*>(idx.data_ptr());
    a.topk_w = static_cast<float*>(weight.data_ptr());
    a.stream = w.stream;
    check(::mok_gate(&a));
    PyObject* out = PyTuple_New(2);
    if (!out) throw python_error();
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(idx)));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(weight)));
    return out;
    END_HANDLE_TH_ERRORS
}

const char GATE_BACKWARD_DOC[] =
    "mok_gate_backward(logits, topk_idx, dw, score='softmax', renormalise=True, scale=1.0, stream=None)\n"
    "--\n\n"
    "dL/dlogits [T, E] (in the logits' type) from dL/dtopk_w (dw) and the chosen experts of mok_gate.\n"
    "In a torch.autograd.Function it is the backward of mok_gate's weights.";
PyObject* gate_backward(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"logits", "topk_idx", "dw", "score", "renormalise", "scale", "stream"};
    static const Names<7> names(texts);
    const Call<7> c("mok_gate_backward", names, 3, args, n, kw);
    const at::Tensor &logits = tensor("logits", c.v[0]), &idx = tensor("topk_idx", c.v[1]);
    const Where w("mok_gate_backward", logits, c.v[6]);
    mok_gate_bwd_args a = {};
    a.logits_stride = rows("logits", logits, 0, w.device);
    a.logits = logits.data_ptr();
    a.logits_type = type_of("logits", logits.scalar_type());
    TORCH_CHECK_VALUE(idx.dim() == 2 && logits.size(0) <= INT32_MAX && logits.size(1) <= INT32_MAX, "topk_idx: expected [T, k]");
    const int64_t T = logits.size(0), k = idx.size(1);
    a.topk_idx = static_cast<const int32_t*>(packed("topk_idx", idx, {T, k}, at::kInt, w.device));
    a.dw = static_cast<const float*>(packed("dw", tensor("dw", c.v[2]), {T, k}, at::kFloat, w.device));
    a.T = (int32_t)T;
    a.E = (int32_t)logits.size(1);
    a.k = (int32_t)k;
    a.score = score(c.v[3]);
    a.renormalise = truth(c.v[4], true);
    a.scale = (float)number(c.v[5], 1.0);
    at::Tensor out = make({T, logits.size(1)}, logits.scalar_type(), w.device);
    a.dlogits = out.data_ptr();
    a.dlogits_stride = logits.size(1);
    a.stream = w.stream;
    check(::mok_gate_backward(&a));
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

const char QUANTIZE_DOC[] =
    "mok_i8_quantize(x, stream=None)\n"
    "--\n\n"
    "Rows of x [..., K] (bf16, fp16 or fp32) -> (codes int8 [..., K rounded up to 16], scales fp32 [...]).";
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"x", "stream"};
    static const Names<2> names(texts);
    const Call<2> c("mok_i8_quantize", names, 1, args, n, kw);
    const at::Tensor& x = tensor("x", c.v[0]);
    const Where w("mok_i8_quantize", x, c.v[1]);
    TORCH_CHECK_VALUE(x.dim() >= 1, "x: expected rows");
    const int64_t K = x.size(-1), pitch = (K + 15) / 16 * 16;
    TORCH_CHECK_VALUE(K <= INT32_MAX, "x: rows too long");
    const at::Tensor flat = x.dim() == 2 ? x : x.reshape({x.numel() / (K > 0 ? K : 1), K});
    const int64_t ldx = rows("x", flat, K, w.device);
    std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = pitch;
    at::Tensor codes = make(shape, at::kChar, w.device);
    shape.pop_back();
    at::Tensor scales = make(shape, at::kFloat, w.device);
    check(::mok_i8_quantize(flat.data_ptr(), type_of("x", x.scalar_type()), flat.size(0), (int)K, ldx,
                            static_cast<int8_t*>(codes.data_ptr()), pitch, static_cast<float*>(scales.data_ptr()), w.stream));
    PyObject* out = PyTuple_New(2);
    if (!out) throw python_error();
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(codes)));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(scales)));
    return out;
    END_HANDLE_TH_ERRORS
}

// The common part of the two products: a.x or a.x_codes and a.K are set.
PyObject* product(mok_i8_linear_args& a, const Weights& weights, int64_t M, int64_t K, PyObject* bias, at::ScalarType out_type,
                  PyObject* workspace, const Where& w) {
    TORCH_CHECK_VALUE(M <= INT32_MAX && K <= INT32_MAX && weights.codes.defined() && weights.codes.dim() == 2 &&
                          weights.codes.scalar_type() == at::kChar && weights.scales.defined() && weights.codes.size(0) <= INT32_MAX,
                      "weights: expected I8Weights with int8 codes [N, K]");
    const int64_t N = weights.codes.size(0);
    a.w_stride = rows("weights.codes", weights.codes, K, w.device);
    a.W_codes = static_cast<const int8_t*>(weights.codes.data_ptr());
    a.W_scales = static_cast<const float*>(packed("weights.scales", weights.scales, {N}, at::kFloat, w.device));
    if (bias) a.bias = static_cast<const float*>(packed("bias", tensor("bias", bias), {N}, at::kFloat, w.device));
    a.M = (int32_t)M;
    a.K = (int32_t)K;
    a.N = (int32_t)N;
    a.out_type = type_of("out_dtype", out_type);
    at::Tensor out = make({M, N}, out_type, w.device), own;
    a.out = out.data_ptr();
    a.out_stride = N;
    a.stream = w.stream;
    scratch(workspace, a.x ? ::mok_i8_linear_workspace_bytes(&a) : 0, w.device, own, &a.workspace, &a.workspace_bytes);
    check(::mok_i8_linear(&a));
    return THPVariable_Wrap(std::move(out));
}

const char LINEAR_DOC[] =
    "mok_i8_linear(x, weights, bias=None, out_dtype=None, workspace=None, stream=None)\n"
    "--\n\n"
    "out [M, N] = quantise(x [M, K]) W8^T (+ bias): the rows of x are quantised in the call.  weights: I8Weights [N, K]; out_dtype\n"
    "defaults to x's.  workspace: a uint8 tensor of M * (K + 20) + 768 bytes (None: allocated if the call needs it).";
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"x", "weights", "bias", "out_dtype", "workspace", "stream"};
    static const Names<6> names(texts);
    const Call<6> c("mok_i8_linear", names, 2, args, n, kw);
    const at::Tensor& x = tensor("x", c.v[0]);
    const Where w("mok_i8_linear", x, c.v[5]);
    mok_i8_linear_args a = {};
    a.x_stride = rows("x", x, 0, w.device);
    a.x = x.data_ptr();
    a.x_type = type_of("x", x.scalar_type());
    return product(a, Weights("weights", c.v[1]), x.size(0), x.size(1), c.v[2], dtype_of(c.v[3], x.scalar_type()), c.v[4], w);
    END_HANDLE_TH_ERRORS
}

const char MATMUL_DOC[] =
    "mok_i8_matmul(codes, scales, weights, K=None, bias=None, out_dtype=torch.bfloat16, stream=None)\n"
    "--\n\n"
    "out [M, N] from rows that are 8-bit already (mok_i8_quantize): codes int8 [M, >= K], scales fp32 [M]; K defaults to the\n"
    "weights' columns.";
PyObject* matmul(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"codes", "scales", "weights", "K", "bias", "out_dtype", "stream"};
    static const Names<7> names(texts);
    const Call<7> c("mok_i8_matmul", names, 3, args, n, kw);
    const at::Tensor& codes = tensor("codes", c.v[0]);
    const Where w("mok_i8_matmul", codes, c.v[6]);
    const Weights weights("weights", c.v[2]);
    TORCH_CHECK_VALUE(weights.codes.defined() && weights.codes.dim() == 2 && codes.dim() == 2 && codes.scalar_type() == at::kChar,
                      "codes: expected int8 [M, K] and weights [N, K]");
    const int64_t K = small("K", c.v[3], weights.codes.size(1));
    mok_i8_linear_args a = {};
    a.codes_stride = rows("codes", codes, K, w.device);
    a.x_codes = static_cast<const int8_t*>(codes.data_ptr());
    a.x_scales = static_cast<const float*>(packed("scales", tensor("scales", c.v[1]), {codes.size(0)}, at::kFloat, w.device));
    return product(a, weights, codes.size(0), K, c.v[4], dtype_of(c.v[5], at::kBFloat16), nullptr, w);
    END_HANDLE_TH_ERRORS
}

// A stack of 8-bit matrices [E, n, >= width]: sets the addresses and the row pitch.
void stack(const char* name, const Weights& m, int64_t E, int64_t n, int64_t width, c10::Device device, const int8_t** codes,
           const float** scales, int64_t* pitch) {
    TORCH_CHECK_VALUE(m.codes.defined() && m.scales.defined() && m.codes.dim() == 3 && m.codes.size(2) >= width, name,
                      ".codes: expected [", E, ", ", n, ", >= ", width, "]");
    *pitch = m.codes.size(2);
    *codes = static_cast<const int8_t*>(packed(name, m.codes, {E, n, *pitch}, at::kChar, device));
    *scales = static_cast<const float*>(packed(name, m.scales, {E, n}, at::kFloat, device));
}

const char EXPERTS_DOC[] =
    "mok_i8_experts(x, topk_idx, topk_w, gate_up, down, add=None, workspace=None, stream=None)\n"
    "--\n\n"
    "out [T, H] = add + sum_s topk_w[:, s] f_{topk_idx[:, s]}(x) on 8-bit operands; gate_up: I8Weights [E, 2I, H], down: I8Weights\n"
    "[E, H, I].  Ids outside 0 .. E-1 are not routed.  workspace: from alloc_i8_workspace (None: allocated).";
PyObject* experts(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"x", "topk_idx", "topk_w", "gate_up", "down", "add", "workspace", "stream"};
    static const Names<8> names(texts);
    const Call<8> c("mok_i8_experts", names, 5, args, n, kw);
    const at::Tensor &x = tensor("x", c.v[0]), &idx = tensor("topk_idx", c.v[1]);
    const Where w("mok_i8_experts", x, c.v[7]);
    const Weights gate_up("gate_up", c.v[3]), down("down", c.v[4]);
    mok_i8_experts_args a = {};
    a.x_stride = rows("x", x, 0, w.device);
    const int64_t T = x.size(0), H = x.size(1);
    TORCH_CHECK_VALUE(x.scalar_type() == at::kBFloat16 || x.scalar_type() == at::kHalf, "x: expected bfloat16 or float16, got ", x.scalar_type());
    TORCH_CHECK_VALUE(idx.dim() == 2, "topk_idx: expected [T, k]");
    TORCH_CHECK_VALUE(gate_up.codes.defined() && gate_up.codes.dim() == 3, "gate_up: expected I8Weights [E, 2I, H]");
    const int64_t k = idx.size(1), E = gate_up.codes.size(0), I = gate_up.codes.size(1) / 2;
    TORCH_CHECK_VALUE(T <= INT32_MAX && H <= INT32_MAX && I <= INT32_MAX && E <= INT32_MAX && k <= INT32_MAX, "x: too large");
    a.x = x.data_ptr();
    a.type = type_of("x", x.scalar_type());
    a.topk_idx = static_cast<const int32_t*>(packed("topk_idx", idx, {T, k}, at::kInt, w.device));
    a.topk_w = static_cast<const float*>(packed("topk_w", tensor("topk_w", c.v[2]), {T, k}, at::kFloat, w.device));
    stack("gate_up", gate_up, E, 2 * I, H, w.device, &a.gate_up_codes, &a.gate_up_scales, &a.gate_up_stride);
    stack("down", down, E, H, I, w.device, &a.down_codes, &a.down_scales, &a.down_stride);
    TORCH_CHECK_VALUE(down.max.defined(), "down.max is missing");
    a.down_max = static_cast<const float*>(packed("down.max", down.max, {E}, at::kFloat, w.device));
    if (c.v[5]) {
        const at::Tensor& add = tensor("add", c.v[5]);
        TORCH_CHECK_VALUE(add.sizes() == x.sizes() && add.scalar_type() == x.scalar_type(), "add: expected ", x.sizes(), " of ",
                          x.scalar_type(), ", got ", add.sizes(), " of ", add.scalar_type());
        a.add_stride = rows("add", add, H, w.device);
        a.add = add.data_ptr();
    }
    a.T = (int32_t)T;
    a.H = (int32_t)H;
    a.I = (int32_t)I;
    a.E = (int32_t)E;
    a.k = (int32_t)k;
    at::Tensor out = make({T, H}, x.scalar_type(), w.device), own;
    a.out = out.data_ptr();
    a.out_stride = H;
    a.stream = w.stream;
    scratch(c.v[6], c.v[6] ? 0 : ::mok_i8_experts_workspace_bytes(a.T, a.H, a.I, a.E, a.k), w.device, own, &a.workspace, &a.workspace_bytes);
    check(::mok_i8_experts(&a));
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

const char FEW_DOC[] =
    "mok_moe_few(x, W_router, router_bias, W_gate_up, W_down, W_shared_gate_up, W_shared_down, k, workspace=None, bias=None,\n"
    "            score='softmax', n_groups=1, topk_groups=1, group_top=2, renormalise=True, scale=1.0, add=None, stages=False, debug=0,\n"
    "            stream=None)\n"
    "--\n\n"
    "The whole layer for up to 64 tokens x [T, H] (bf16 or fp16) in one launch; routing as in mok_gate, add [T, H] is added to the\n"
    "output.  Returns out [T, H], or (out, topk_idx, topk_w) with stages.  workspace: from alloc_few_workspace (None: allocated).\n"
    "Outside of autograd, like the layer's own calls.";
PyObject* few(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"x", "W_router", "router_bias", "W_gate_up", "W_down", "W_shared_gate_up", "W_shared_down", "k",
                                        "workspace", "bias", "score", "n_groups", "topk_groups", "group_top", "renormalise", "scale",
                                        "add", "stages", "debug", "stream"};
    static const Names<20> names(texts);
    const Call<20> c("mok_moe_few", names, 0, args, n, kw);
    for (int i : {0, 1, 3, 4, 7})
        if (!c.v[i]) c.throw_type("mok_moe_few", std::string("missing argument ") + texts[i]);
    const at::Tensor &x = tensor("x", c.v[0]), &router = tensor("W_router", c.v[1]), &gate_up = tensor("W_gate_up", c.v[3]);
    const Where w("mok_moe_few", x, c.v[19]);
    TORCH_CHECK_VALUE(x.scalar_type() == at::kBFloat16 || x.scalar_type() == at::kHalf, "x: expected bfloat16 or float16, got ", x.scalar_type());
    mok_few_args a = {};
    a.x_stride = rows("x", x, 0, w.device);
    const int64_t T = x.size(0), H = x.size(1);
    TORCH_CHECK_VALUE(router.dim() == 2 && gate_up.dim() == 3, "W_router: expected [E, H], W_gate_up: [E, 2I, H]");
    const int64_t E = router.size(0), I = gate_up.size(1) / 2;
    TORCH_CHECK_VALUE(T <= INT32_MAX && H <= INT32_MAX && E <= INT32_MAX && I <= INT32_MAX, "x: too large");
    const at::ScalarType type = x.scalar_type();
    a.x = x.data_ptr();
    a.type = type_of("x", type);
    a.W_router = static_cast<const float*>(packed("W_router", router, {E, H}, at::kFloat, w.device));
    if (c.v[2]) a.router_bias = static_cast<const float*>(packed("router_bias", tensor("router_bias", c.v[2]), {E}, at::kFloat, w.device));
    a.W_gate_up = packed("W_gate_up", gate_up, {E, 2 * I, H}, type, w.device);
    a.W_down = packed("W_down", tensor("W_down", c.v[4]), {E, H, I}, type, w.device);
    if (c.v[5]) {
        const at::Tensor& shared = tensor("W_shared_gate_up", c.v[5]);
        TORCH_CHECK_VALUE(shared.dim() == 2 && shared.size(0) > 0 && shared.size(0) <= INT32_MAX, "W_shared_gate_up: expected [2 I_shared, H]");
        a.I_shared = (int32_t)(shared.size(0) / 2);
        a.W_shared_gate_up = packed("W_shared_gate_up", shared, {2 * (int64_t)a.I_shared, H}, type, w.device);
    }
    if (c.v[6]) a.W_shared_down = packed("W_shared_down", tensor("W_shared_down", c.v[6]), {H, a.I_shared}, type, w.device);
    a.k = small("k", c.v[7], 0);
    if (c.v[9]) a.bias = static_cast<const float*>(packed("bias", tensor("bias", c.v[9]), {E}, at::kFloat, w.device));
    a.score = score(c.v[10]);
    a.n_groups = small("n_groups", c.v[11], 1);
    a.topk_groups = small("topk_groups", c.v[12], 1);
    a.group_top = small("group_top", c.v[13], 2);
    a.renormalise = truth(c.v[14], true);
    a.scale = (float)number(c.v[15], 1.0);
    if (c.v[16]) {
        const at::Tensor& add = tensor("add", c.v[16]);
        TORCH_CHECK_VALUE(add.sizes() == x.sizes() && add.scalar_type() == type, "add: expected ", x.sizes(), " of ", type, ", got ",
                          add.sizes(), " of ", add.scalar_type());
        a.add_stride = rows("add", add, H, w.device);
        a.add = add.data_ptr();
    }
    a.T = (int32_t)T;
    a.H = (int32_t)H;
    a.I = (int32_t)I;
    a.E = (int32_t)E;
    const size_t need = ::mok_few_workspace_bytes(a.T, a.H, a.I, a.I_shared, a.E, a.k);
    if (!need) check(MOK_ERR_SHAPE);                     // (before outputs of that size are allocated)
    const bool stages = truth(c.v[17], false);
    a.debug = small("debug", c.v[18], 0);
    at::Tensor out = make({T, H}, type, w.device), idx, weight, own;
    a.out = out.data_ptr();
    a.out_stride = H;
    if (stages) {
        idx = make({T, a.k}, at::kInt, w.device);
        weight = make({T, a.k}, at::kFloat, w.device);
        a.topk_idx = static_cast<int32_t*>(idx.data_ptr());
        a.topk_w = static_cast<float*>(weight.data_ptr());
    }
    a.stream = w.stream;
    scratch(c.v[8], need, w.device, own, &a.workspace, &a.workspace_bytes);
    check(::mok_moe_few(&a));
    if (!stages) return THPVariable_Wrap(std::move(out));
    PyObject* all = PyTuple_New(3);
    if (!all) throw python_error();
    PyTuple_SET_ITEM(all, 0, THPVariable_Wrap(std::move(out)));
    PyTuple_SET_ITEM(all, 1, THPVariable_Wrap(std::move(idx)));
    PyTuple_SET_ITEM(all, 2, THPVariable_Wrap(std::move(weight)));
    return all;
    END_HANDLE_TH_ERRORS
}

// The arguments that mok_block_join and its gradient share, from `first` on.
#define JOIN_RULE "before", "before_weight", "before_bias", "after", "after_weight", "after_bias", "gate", "scale", "eps", "p", "seed", "offset"
int32_t norm(const char* name, PyObject* o) {
    if (!o) return MOK_NORM_NONE;
    TORCH_CHECK_TYPE(PyUnicode_Check(o), name, ": expected a string or None");
    if (PyUnicode_CompareWithASCIIString(o, "rms") == 0) return MOK_NORM_RMS;
    if (PyUnicode_CompareWithASCIIString(o, "layer") == 0) return MOK_NORM_LAYER;
    TORCH_CHECK_VALUE(false, name, ": expected \"rms\", \"layer\" or None, got \"", text(o), "\"");
}
// A 64-bit word from any Python integer, as the language itself would wrap it
uint64_t word(PyObject* o) {
    if (!o) return 0;
    const unsigned long long r = PyLong_AsUnsignedLongLongMask(o);
    if (r == (unsigned long long)-1 && PyErr_Occurred()) throw python_error();
    return r;
}
void join_rule(mok_join_args& a, PyObject* const* v, const at::Tensor* x, const at::Tensor* y, const at::Tensor& rows_of, c10::Device device) {
    TORCH_CHECK_VALUE(rows_of.dim() == 2 && rows_of.size(0) <= INT32_MAX && rows_of.size(1) <= INT32_MAX, "expected matrices [T, H]");
    const int64_t T = rows_of.size(0), H = rows_of.size(1);
    a.T = (int32_t)T;
    a.H = (int32_t)H;
    auto matrix = [&](const char* name, const at::Tensor& t, at::ScalarType type) {
        TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == T && t.size(1) == H && t.scalar_type() == type, name, ": expected [", T, ", ", H, "] of ", type,
                          ", got ", t.sizes(), " of ", t.scalar_type());
        return rows(name, t, H, device);
    };
    const at::ScalarType type = y ? y->scalar_type() : rows_of.scalar_type(), stream = x ? x->scalar_type() : type;
    a.type = type_of("y", type);
    a.x_type = type_of("x", stream);
    if (x) {
        a.x_stride = matrix("x", *x, stream);
        a.x = x->data_ptr();
    }
    if (y) {
        a.y_stride = matrix("y", *y, type);
        a.y = y->data_ptr();
    }
    a.before = norm("before", v[0]);
    a.after = norm("after", v[3]);
    TORCH_CHECK_VALUE((a.before || (!v[1] && !v[2])) && (a.after || (!v[4] && !v[5])), "a norm's weight or bias without the norm");
    at::ScalarType vectors = at::kFloat;
    bool known = false;
    auto vector = [&](const char* name, PyObject* o) -> const void* {
        if (!o) return nullptr;
        const at::Tensor& t = tensor(name, o);
        if (!known) vectors = t.scalar_type();
        known = true;
        return packed(name, t, {H}, vectors, device);
    };
    a.before_weight = vector("before_weight", v[1]);
    a.before_bias = vector("before_bias", v[2]);
    a.after_weight = vector("after_weight", v[4]);
    a.after_bias = vector("after_bias", v[5]);
    if (v[6]) {
        const at::Tensor& gate = tensor("gate", v[6]);
        if (gate.dim() == 1) {
            a.gate_kind = MOK_JOIN_GATE_CHANNEL;
            a.gate = vector("gate", v[6]);
        } else {
            TORCH_CHECK_VALUE(gate.dim() == 2 && gate.size(0) == T && (gate.size(1) == H || gate.size(1) == 1) && gate.scalar_type() == type &&
                                  gate.device() == device, "gate: expected [H], or [T, 1] or [T, H] of ", type, " on ", device, ", got ", gate.sizes(),
                              " of ", gate.scalar_type(), " on ", gate.device());
            a.gate_kind = gate.size(1) == H && H > 1 ? MOK_JOIN_GATE_FULL : MOK_JOIN_GATE_TOKEN;
            if (a.gate_kind == MOK_JOIN_GATE_FULL) a.gate_stride = rows("gate", gate, H, device);
            else a.gate_stride = T > 1 ? gate.stride(0) : 1;
            a.gate = gate.data_ptr();
        }
    }
    a.vector_type = type_of("vectors", vectors);
    a.scale = (float)number(v[7], 1.0);
    a.eps = (float)number(v[8], 1e-6);
    a.p = number(v[9], 0.0);
    if (v[10] && THPVariable_Check(v[10])) {             // {seed, offset} on the device
        const at::Tensor& at = THPVariable_Unpack(v[10]);
        TORCH_CHECK_VALUE(!v[11], "offset: is the second element of a seed tensor");
        a.seed_at = static_cast<const uint64_t*>(packed("seed", at, {2}, at::kLong, device));
    } else {
        a.seed = word(v[10]);
        a.offset = word(v[11]);
    }
}
const at::Tensor* maybe(const char* name, PyObject* o) { return o ? &tensor(name, o) : nullptr; }
PyObject* wrap_or_none(at::Tensor&& t) {
    if (t.defined()) return THPVariable_Wrap(std::move(t));
    Py_RETURN_NONE;
}

const char JOIN_DOC[] =
    "mok_block_join(x, y=None, before=None, before_weight=None, before_bias=None, after=None, after_weight=None, after_bias=None,\n"
    "               gate=None, scale=1.0, eps=1e-6, p=0.0, seed=0, offset=0, dtype=None, stream=None)\n"
    "--\n\n"
    "(sum, normed): sum = x + scale * drop(gate * norm_after(y)), normed = norm_before(sum), rows [T, H] of bf16, fp16 or fp32; x may be\n"
    "fp32 beside any y, or None (nothing is added to).  before, after: 'rms', 'layer' or None (normed is then None).  gate: [H], [T, 1]\n"
    "or [T, H].  p: probability of dropping an element; seed, offset: integers, or seed an int64 tensor [2] of both on the device, which\n"
    "a captured call reads on every replay.  Without y, sum is x itself, and normed may be of another dtype.  Outside of autograd:\n"
    "gradients come from mok_block_join_backward.";
PyObject* join(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"x", "y", JOIN_RULE, "dtype", "stream"};
    static const Names<16> names(texts);
    const Call<16> c("mok_block_join", names, 0, args, n, kw);
    const at::Tensor *x = maybe("x", c.v[0]), *y = maybe("y", c.v[1]);
    if (!x && !y) c.throw_type("mok_block_join", "missing argument x or y");
    const at::Tensor& first = x ? *x : *y;
    const Where w("mok_block_join", first, c.v[15]);
    mok_join_args a = {};
    join_rule(a, c.v + 2, x, y, first, w.device);
    TORCH_CHECK_VALUE(y || (!a.after && !a.gate_kind), "after, gate: there is no y");
    at::Tensor sum, normed;
    at::ScalarType of = y ? y->scalar_type() : x->scalar_type();
    if (c.v[14]) {                                       // the type of normed where no y says it
        TORCH_CHECK_TYPE(THPDtype_Check(c.v[14]), "dtype: expected a torch.dtype");
        TORCH_CHECK_VALUE(!y, "dtype: normed is of y's type");
        of = reinterpret_cast<THPDtype*>(c.v[14])->scalar_type;
        a.type = type_of("dtype", of);
    }
    if (a.H < 1 || a.H > MOK_JOIN_MAX_WIDTH) check(MOK_ERR_SHAPE);
    if (y) {
        sum = make({a.T, a.H}, x ? x->scalar_type() : y->scalar_type(), w.device);
        a.sum = sum.data_ptr();
        a.sum_stride = a.H;
    }
    if (a.before) {
        normed = make({a.T, a.H}, of, w.device);
        a.normed = normed.data_ptr();
        a.normed_stride = a.H;
    }
    a.stream = w.stream;
    check(::mok_block_join(&a));
    PyObject* out = PyTuple_New(2);
    if (!out) throw python_error();
    if (!y) Py_INCREF(c.v[0]);
    PyTuple_SET_ITEM(out, 0, y ? THPVariable_Wrap(std::move(sum)) : c.v[0]);
    PyTuple_SET_ITEM(out, 1, wrap_or_none(std::move(normed)));
    return out;
    END_HANDLE_TH_ERRORS
}

const char JOIN_BACKWARD_DOC[] =
    "mok_block_join_backward(d_sum, d_normed, sum, y=None, before=None, before_weight=None, before_bias=None, after=None,\n"
    "                        after_weight=None, after_bias=None, gate=None, scale=1.0, eps=1e-6, p=0.0, seed=0, offset=0,\n"
    "                        workspace=None, stream=None)\n"
    "--\n\n"
    "(dx, dy, dgate, dbefore_weight, dbefore_bias, dafter_weight, dafter_bias) of mok_block_join, None for what there is not: from the\n"
    "gradients of its outputs (d_sum may be None: 0), the sum that it returned (None is enough without `before`), y and its other\n"
    "arguments.  The gradients of vectors are fp32.  y=None: those of sum and before only.";
PyObject* join_backward(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    HANDLE_TH_ERRORS
    static const char* const texts[] = {"d_sum", "d_normed", "sum", "y", JOIN_RULE, "workspace", "stream"};
    static const Names<18> names(texts);
    const Call<18> c("mok_block_join_backward", names, 0, args, n, kw);
    const at::Tensor *d_sum = maybe("d_sum", c.v[0]), *d_normed = maybe("d_normed", c.v[1]), *sum = maybe("sum", c.v[2]), *y = maybe("y", c.v[3]);
    if (!d_sum && !d_normed) c.throw_type("mok_block_join_backward", "missing argument d_sum or d_normed");
    const at::Tensor& first = d_sum ? *d_sum : *d_normed;
    const Where w("mok_block_join_backward", first, c.v[17]);
    mok_join_bwd_args b = {};
    mok_join_args& a = b.forward;
    join_rule(a, c.v + 4, sum ? sum : d_sum, y ? y : d_normed, first, w.device);
    if (!sum) a.x = nullptr;
    if (!y) a.y = nullptr;
    TORCH_CHECK_VALUE(y || (!a.after && !a.gate_kind), "after, gate: there is no y");
    TORCH_CHECK_VALUE((d_normed != nullptr) == (a.before != 0) && (!a.before || sum), "d_normed and sum belong to a norm before");
    const at::ScalarType type = (y ? *y : d_normed ? *d_normed : first).scalar_type(), stream = (sum ? *sum : d_sum ? *d_sum : first).scalar_type();
    auto matrix = [&](const char* name, const at::Tensor& t, at::ScalarType of) {
        TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == a.T && t.size(1) == a.H && t.scalar_type() == of, name, ": expected [", a.T, ", ", a.H, "] of ",
                          of, ", got ", t.sizes(), " of ", t.scalar_type());
        return rows(name, t, a.H, w.device);
    };
    if (d_sum) {
        b.d_sum_stride = matrix("d_sum", *d_sum, stream);
        b.d_sum = d_sum->data_ptr();
    }
    if (d_normed) {
        b.d_normed_stride = matrix("d_normed", *d_normed, type);
        b.d_normed = d_normed->data_ptr();
    }
    if (a.H < 1 || a.H > MOK_JOIN_MAX_WIDTH) check(MOK_ERR_SHAPE);
    at::Tensor out[7], own;
    out[0] = make({a.T, a.H}, stream, w.device);
    b.dx = out[0].data_ptr();
    b.dx_stride = a.H;
    if (y) {
        out[1] = make({a.T, a.H}, type, w.device);
        b.dy = out[1].data_ptr();
        b.dy_stride = a.H;
    }
    if (a.gate_kind) {
        const int64_t width = a.gate_kind == MOK_JOIN_GATE_TOKEN ? 1 : a.H;
        out[2] = a.gate_kind == MOK_JOIN_GATE_CHANNEL ? make({a.H}, at::kFloat, w.device) : make({a.T, width}, type, w.device);
        b.dgate = out[2].data_ptr();
        b.dgate_stride = width;
    }
    float** const vectors[4] = {&b.d_before_weight, &b.d_before_bias, &b.d_after_weight, &b.d_after_bias};
    const void* const given[4] = {a.before_weight, a.before_bias, a.after_weight, a.after_bias};
    bool sums = a.gate_kind == MOK_JOIN_GATE_CHANNEL;
    for (int i = 0; i < 4; ++i)
        if (given[i]) {
            out[3 + i] = make({a.H}, at::kFloat, w.device);
            *vectors[i] = static_cast<float*>(out[3 + i].data_ptr());
            sums = true;
        }
    scratch(c.v[16], sums ? ::mok_join_bwd_workspace_bytes(a.T, a.H) : 0, w.device, own, &b.workspace, &b.workspace_bytes);
    b.stream = w.stream;
    check(::mok_block_join_backward(&b));
    PyObject* all = PyTuple_New(7);
    if (!all) throw python_error();
    for (int i = 0; i < 7; ++i) PyTuple_SET_ITEM(all, i, wrap_or_none(std::move(out[i])));
    return all;
    END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* error) {
    Py_XINCREF(error);
    Py_XSETREF(g_error, error);
    Py_RETURN_NONE;
}

#define MOK_FAST(name, function, doc) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(function)), METH_FASTCALL | METH_KEYWORDS, doc}
PyMethodDef methods[] = {MOK_FAST("mok_gate", gate, GATE_DOC),
                         MOK_FAST("mok_gate_backward", gate_backward, GATE_BACKWARD_DOC),
                         MOK_FAST("mok_i8_quantize", quantize, QUANTIZE_DOC),
                         MOK_FAST("mok_i8_linear", linear, LINEAR_DOC),
                         MOK_FAST("mok_i8_matmul", matmul, MATMUL_DOC),
                         MOK_FAST("mok_i8_experts", experts, EXPERTS_DOC),
                         MOK_FAST("mok_moe_few", few, FEW_DOC),
                         MOK_FAST("mok_block_join", join, JOIN_DOC),
                         MOK_FAST("mok_block_join_backward", join_backward, JOIN_BACKWARD_DOC),
                         {"set_error", set_error, METH_O, "The exception class that a refused call raises (called with the status)."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Entry points of libmok for torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
