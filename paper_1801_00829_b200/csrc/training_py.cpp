// CPython extension behind training.py: argument checks and marshalling of calls that are made once per layer or step and
// for small inputs take less time on the GPU than a call assembled in Python takes on the host (block norm 15 us, its
// gradient 30, clipping and AdamW 13 to 16; here 7, 12 and less than the GPU takes).  Nothing here computes.
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <map>
#include <string>
#include <utility>

#include "fusedops_train.h"

namespace {

PyObject *g_error = nullptr;        // FusedOpsError
PyObject *g_workspace = nullptr;    // f(GPU number, bytes) -> tensor: the current stream's scratch

struct Refused : std::exception {
    std::string text;
    explicit Refused(std::string t) : text(std::move(t)) {}
    const char *what() const noexcept override { return text.c_str(); }
};
struct Raised : std::exception {};   // a Python exception is set

void require(bool ok, const char *text)
{
    if (!ok) throw Refused(text);
}

int type_code(at::ScalarType t)
{
    switch (t) {
    case at::kDouble: return FO_F64;
    case at::kFloat: return FO_F32;
    case at::kBFloat16: return FO_BF16;
    case at::kHalf: return FO_F16;
    default: throw Refused(std::string("no kernel for ") + c10::toString(t));
    }
}

const at::Tensor *tensor_of(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Refused(std::string(name) + " is not a tensor");
    return &THPVariable_Unpack(o);
}

// What every matrix and vector of one call has to agree with.
struct Call {
    int64_t rows, cols;
    c10::DeviceIndex gpu;

    explicit Call(const at::Tensor &like)
    {
        require(like.is_cuda(), "fused operators need CUDA tensors (no CPU path)");
        require(like.dim() == 2, "matrices are 2-D");
        rows = like.size(0), cols = like.size(1), gpu = like.get_device();
    }
    [[noreturn]] void refuse(const at::Tensor &t, const char *name, const char *what, at::ScalarType type) const
    {
        std::string s = std::string(name) + ": " + what + " of " + c10::toString(type) + " on GPU "
                        + std::to_string((int)gpu) + " is needed, not " + c10::toString(t.scalar_type()) + " [";
        for (int64_t n : t.sizes()) s += " " + std::to_string(n);
        throw Refused(s + " ] on " + t.device().str());
    }
    void *matrix(const at::Tensor *t, at::ScalarType type, const char *name, int64_t *ld) const
    {
        *ld = 0;
        if (!t) return nullptr;
        if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || t->scalar_type() != type || !t->is_cuda()
            || t->get_device() != gpu)
            refuse(*t, name, "a matrix of the call's shape", type);
        if (cols > 1 && t->stride(1) != 1) throw Refused(std::string("rows of ") + name + " must be contiguous");
        *ld = t->stride(0);
        if (*ld < cols) {
            if (rows > 1) throw Refused(std::string("rows of ") + name + " overlap");
            *ld = cols;
        }
        return t->data_ptr();
    }
    void *vector(const at::Tensor *t, at::ScalarType type, const char *name) const
    {
        if (!t) return nullptr;
        if (t->dim() != 1 || t->size(0) != cols || t->scalar_type() != type || !t->is_cuda() || t->get_device() != gpu
            || !t->is_contiguous())
            refuse(*t, name, "a contiguous vector over the columns", type);
        return t->data_ptr();
    }
    at::Tensor make(at::IntArrayRef sizes, at::ScalarType type) const
    {
        return at::detail::empty_cuda(sizes, type, c10::Device(c10::kCUDA, gpu), c10::nullopt);
    }
};

bool is(PyObject *o, const char *text) { return PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, text) == 0; }

// (kind, weight, bias, eps) or None
struct Norm {
    const at::Tensor *weight = nullptr, *bias = nullptr;
    fo_norm c = {};
    explicit Norm(PyObject *o)
    {
        if (o == Py_None) return;
        require(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 4, "a norm is (kind, weight, bias, eps)");
        PyObject *kind = PyTuple_GET_ITEM(o, 0);
        c.kind = is(kind, "rms") ? FO_NORM_RMS : is(kind, "layer") ? FO_NORM_LAYER : FO_NORM_NONE;
        require(c.kind != FO_NORM_NONE, "a norm is \"rms\" or \"layer\"");
        weight = tensor_of(PyTuple_GET_ITEM(o, 1), "weight");
        bias = tensor_of(PyTuple_GET_ITEM(o, 2), "bias");
        c.eps = PyFloat_AsDouble(PyTuple_GET_ITEM(o, 3));
        if (PyErr_Occurred()) throw Raised();
    }
    bool given() const { return c.kind != FO_NORM_NONE; }
    void check(const Call &call, at::ScalarType type, const char *name)
    {
        c.weight = call.vector(weight, type, name);
        c.bias = call.vector(bias, type, name);
    }
};

// (access, tensor, activation) or None
struct Gate {
    const at::Tensor *t = nullptr;
    int access = 0, act = 0;
    void *p = nullptr;
    int64_t ld = 0;
    explicit Gate(PyObject *o)
    {
        if (o == Py_None) return;
        require(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 3, "a gate is (access, tensor, activation)");
        PyObject *where = PyTuple_GET_ITEM(o, 0), *how = PyTuple_GET_ITEM(o, 2);
        access = is(where, "cell") ? FO_AT_CELL : is(where, "row") ? FO_AT_ROW : is(where, "col") ? FO_AT_COL : -1;
        act = is(how, "linear") ? FO_ACT_LINEAR : is(how, "sigmoid") ? FO_ACT_SIGMOID : is(how, "silu") ? FO_ACT_SILU
              : is(how, "tanh") ? FO_ACT_TANH : -1;
        require(access >= 0, "a gate's access is \"cell\", \"row\" or \"col\"");
        require(act >= 0, "a gate's activation is \"linear\", \"sigmoid\", \"silu\" or \"tanh\"");
        t = tensor_of(PyTuple_GET_ITEM(o, 1), "gate");
        require(t != nullptr, "the gate's tensor is None");
    }
    void check(const Call &call, at::ScalarType type)
    {
        if (!t) return;
        if (access == FO_AT_CELL) {
            p = call.matrix(t, type, "gate", &ld);
            return;
        }
        // a vector, or a matrix of one column (per row) or one row (per column)
        const int64_t n = access == FO_AT_ROW ? call.rows : call.cols;
        const int along = t->dim() == 2 && access == FO_AT_COL ? 1 : 0;
        const bool shaped = t->dim() == 1 || (t->dim() == 2 && t->size(1 - along) == 1);
        if (!shaped || t->size(along) != n || t->scalar_type() != type || !t->is_cuda() || t->get_device() != call.gpu)
            call.refuse(*t, "gate", access == FO_AT_ROW ? "a vector over the rows" : "a vector over the columns", type);
        ld = n > 1 ? t->stride(along) : 1;
        require(access == FO_AT_ROW ? ld >= 1 : ld == 1, "stride of the gate");
        p = t->data_ptr();
    }
};

// The vectors' type is that of the first one given, or the block's; all are checked against it.
at::ScalarType vector_type(at::ScalarType block, const Norm &post, const Norm &pre, const at::Tensor *col_scale)
{
    for (const at::Tensor *t : {col_scale, post.weight, post.bias, pre.weight, pre.bias})
        if (t) return t->scalar_type();
    return block;
}

at::ScalarType sum_type(at::ScalarType block) { return block == at::kDouble ? at::kDouble : at::kFloat; }

// Makes GPU `gpu` current for a call if another one is.
struct OnGpu {
    c10::DeviceIndex before;
    explicit OnGpu(c10::DeviceIndex gpu) : before(c10::cuda::current_device())
    {
        if (gpu == before) before = -1;
        else c10::cuda::set_device(gpu);
    }
    ~OnGpu()
    {
        if (before >= 0) c10::cuda::set_device(before);
    }
};

void check_status(int status, const char *name)
{
    if (status == FO_OK) return;
    PyObject *args = Py_BuildValue("(is)", status, name);
    PyObject *e = args ? PyObject_CallObject(g_error, args) : nullptr;
    Py_XDECREF(args);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Raised();
}

PyObject *or_none(const at::Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

// block_norm(x, f, post, gate, scale, col_scale, pre, out_h, out_y, stats, block_type)
PyObject *block_norm_impl(PyObject *const *a)
{
    const at::Tensor *x = tensor_of(a[0], "x"), *f = tensor_of(a[1], "f"), *col_scale = tensor_of(a[5], "col_scale");
    const at::Tensor *out_h = tensor_of(a[7], "out_h"), *out_y = tensor_of(a[8], "out_y");
    require(x || f, "x or f is needed");
    const at::Tensor &first = x ? *x : *f;
    const Call call(first);
    Norm post(a[2]), pre(a[6]);
    Gate gate(a[3]);
    const double scale = PyFloat_AsDouble(a[4]);
    const int want_stats = PyObject_IsTrue(a[9]);
    if (PyErr_Occurred()) throw Raised();
    const at::ScalarType stream = x || !out_h ? first.scalar_type() : out_h->scalar_type();
    at::ScalarType block = f ? f->scalar_type() : out_y ? out_y->scalar_type() : stream;
    if (!f) {
        require(!post.given() && !gate.t && !col_scale, "post, gate and col_scale need a block output f");
        if (a[10] != Py_None) {
            require(THPDtype_Check(a[10]), "block_type is not a dtype");
            block = reinterpret_cast<THPDtype *>(a[10])->scalar_type;
        } else if (!out_y && stream == at::kFloat) {
            block = vector_type(block, post, pre, col_scale);       // 16-bit weights: the next block's type
        }
    }
    require(!out_y || pre.given(), "out_y without a norm before the next block");
    const at::ScalarType vec = vector_type(block, post, pre, col_scale);

    fo_block_norm n = {};
    n.rows = call.rows, n.cols = call.cols;
    n.stream_type = type_code(stream), n.block_type = type_code(block), n.vec_type = type_code(vec);
    require(stream == block || (stream == at::kFloat && (block == at::kBFloat16 || block == at::kHalf)),
            "no kernel for this pair of stream and block types");
    require(vec == block || (vec == at::kFloat && (block == at::kBFloat16 || block == at::kHalf)),
            "weights, biases and col_scale have the block's type, or float32 beside 16 bits");
    n.x = call.matrix(x, stream, "x", &n.ld_x);
    n.f = call.matrix(f, block, "f", &n.ld_f);
    gate.check(call, block);
    n.gate = gate.p, n.ld_gate = gate.ld, n.gate_access = gate.access, n.gate_act = gate.act;
    n.col_scale = call.vector(col_scale, vec, "col_scale");
    post.check(call, vec, "post"), pre.check(call, vec, "pre");
    n.post = post.c, n.pre = pre.c, n.scale = scale;

    at::Tensor h, y, stats;
    if (out_h) h = *out_h;
    else if (f) h = call.make({call.rows, call.cols}, stream);
    if (out_y) y = *out_y;
    else if (pre.given()) y = call.make({call.rows, call.cols}, block);
    if (want_stats) {
        stats = call.make({4, call.rows}, sum_type(block));
        n.stats = stats.data_ptr();
    }
    n.h = call.matrix(h.defined() ? &h : nullptr, stream, "out_h", &n.ld_h);
    n.y = call.matrix(y.defined() ? &y : nullptr, block, "out_y", &n.ld_y);
    if (n.h || n.y || n.stats) {
        const OnGpu on(call.gpu);
        check_status(fused_block_norm(&n, c10::cuda::getCurrentCUDAStream(call.gpu).stream()), "fused_block_norm");
    }
    PyObject *ho;
    if (h.defined()) {
        ho = out_h ? (Py_INCREF(a[7]), a[7]) : THPVariable_Wrap(h);
    } else {
        ho = (Py_INCREF(a[0]), a[0]);
    }
    PyObject *yo = out_y ? (Py_INCREF(a[8]), a[8]) : or_none(y);
    PyObject *so = or_none(stats), *out = ho && yo && so ? PyTuple_Pack(3, ho, yo, so) : nullptr;
    Py_XDECREF(ho), Py_XDECREF(yo), Py_XDECREF(so);
    return out;
}

at::Tensor workspace(c10::DeviceIndex gpu, cudaStream_t stream, size_t bytes)
{
    static auto *cache = new std::map<std::pair<int, cudaStream_t>, at::Tensor>();      // outlives the interpreter
    at::Tensor &buf = (*cache)[{gpu, stream}];
    if (!buf.defined() || (size_t)buf.numel() < bytes) {
        PyObject *o = PyObject_CallFunction(g_workspace, "in", (int)gpu, (Py_ssize_t)bytes);
        if (!o) throw Raised();
        buf = THPVariable_Unpack(o);
        Py_DECREF(o);
    }
    return buf;
}

// block_norm_grad(dh, dy, h, f, stats, post, gate, scale, col_scale, pre, residual)
PyObject *block_norm_grad_impl(PyObject *const *a)
{
    const at::Tensor *dh = tensor_of(a[0], "dh"), *dy = tensor_of(a[1], "dy"), *h = tensor_of(a[2], "h"), *f = tensor_of(a[3], "f");
    const at::Tensor *stats = tensor_of(a[4], "stats"), *col_scale = tensor_of(a[8], "col_scale");
    require(dh || dy, "dh or dy is needed");
    const Call call(dh ? *dh : *dy);
    Norm post(a[5]), pre(a[9]);
    Gate gate(a[6]);
    const double scale = PyFloat_AsDouble(a[7]);
    const int residual = PyObject_IsTrue(a[10]);
    if (PyErr_Occurred()) throw Raised();
    if (dy) require(pre.given() && h, "dy needs `pre` and h");
    require(f || (!post.given() && !gate.t && !col_scale), "post, gate and col_scale need a block output f");
    const at::ScalarType stream = (dh ? dh : h)->scalar_type();
    const at::ScalarType block = f ? f->scalar_type() : dy ? dy->scalar_type() : stream;
    const at::ScalarType vec = vector_type(block, post, pre, col_scale), sums = sum_type(block);

    fo_block_norm_grad n = {};
    n.rows = call.rows, n.cols = call.cols;
    n.stream_type = type_code(stream), n.block_type = type_code(block), n.vec_type = type_code(vec);
    require(stream == block || (stream == at::kFloat && (block == at::kBFloat16 || block == at::kHalf)),
            "no kernel for this pair of stream and block types");
    require(vec == block || (vec == at::kFloat && (block == at::kBFloat16 || block == at::kHalf)),
            "weights, biases and col_scale have the block's type, or float32 beside 16 bits");
    n.dh = call.matrix(dh, stream, "dh", &n.ld_dh);
    n.dy = call.matrix(dy, block, "dy", &n.ld_dy);
    n.h = call.matrix(dy ? h : nullptr, stream, "h", &n.ld_h);
    n.f = call.matrix(f, block, "f", &n.ld_f);
    gate.check(call, block);
    n.gate = gate.p, n.ld_gate = gate.ld, n.gate_access = gate.access, n.gate_act = gate.act;
    n.col_scale = call.vector(col_scale, vec, "col_scale");
    post.check(call, vec, "post"), pre.check(call, vec, "pre");
    n.post = post.c, n.pre = pre.c, n.scale = scale;
    if (stats) {
        if (stats->dim() != 2 || stats->size(0) != 4 || stats->size(1) != call.rows || stats->scalar_type() != sums
            || !stats->is_contiguous() || !stats->is_cuda() || stats->get_device() != call.gpu)
            call.refuse(*stats, "stats", "4 x rows", sums);
        n.stats = stats->data_ptr();
    }

    PyObject *got = PyDict_New();
    if (!got) throw Raised();
    try {
        auto put = [&](const char *name, at::IntArrayRef sizes, at::ScalarType type) -> void * {
            const at::Tensor t = call.make(sizes, type);
            void *p = t.data_ptr();
            PyObject *o = THPVariable_Wrap(t);
            const int rc = o ? PyDict_SetItemString(got, name, o) : -1;
            Py_XDECREF(o);
            if (rc != 0) throw Raised();
            return p;
        };
        const int64_t cells[2] = {call.rows, call.cols}, cols[1] = {call.cols};
        n.ld_dx = n.ld_df = n.ld_dgate = call.cols;
        if (residual || !f) n.dx = put("x", cells, stream);
        if (f) n.df = put("f", cells, block);
        if (gate.t) n.dgate = put("gate", gate.t->sizes(), gate.access == FO_AT_CELL ? block : sums);
        if (col_scale) n.dcol_scale = put("col_scale", cols, sums);
        if (post.weight) n.dpost_weight = put("post_w", cols, sums);
        if (post.bias) n.dpost_bias = put("post_b", cols, sums);
        if (pre.weight) n.dpre_weight = put("pre_w", cols, sums);
        if (pre.bias) n.dpre_bias = put("pre_b", cols, sums);
        const size_t need = fused_block_norm_grad_workspace_bytes(call.rows, call.cols, n.block_type);
        const OnGpu on(call.gpu);
        const cudaStream_t st = c10::cuda::getCurrentCUDAStream(call.gpu).stream();
        const at::Tensor ws = workspace(call.gpu, st, need);
        check_status(fused_block_norm_grad(&n, ws.data_ptr(), (size_t)ws.numel(), st), "fused_block_norm_grad");
    } catch (...) {
        Py_DECREF(got);
        throw;
    }
    return got;
}

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw Raised();
    return v;
}
long long whole(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) throw Raised();
    return v;
}
// The C structs of a list, packed by training.py
template <class Tensor>
const Tensor *packed_list(PyObject *o, int *count)
{
    require(PyBytes_Check(o) && PyBytes_GET_SIZE(o) % (Py_ssize_t)sizeof(Tensor) == 0, "not a packed list");
    *count = (int)(PyBytes_GET_SIZE(o) / (Py_ssize_t)sizeof(Tensor));
    return reinterpret_cast<const Tensor *>(PyBytes_AS_STRING(o));
}

// grad_norm(list, clip, in_type, out_type, norm_kind, max_norm, eps, result_type, gpu) -> (norm, factor)
PyObject *grad_norm_impl(PyObject *const *a)
{
    int count;
    const fo_tensor *list = packed_list<fo_tensor>(a[0], &count);
    const bool clip = PyObject_IsTrue(a[1]) == 1;
    const int in_type = (int)whole(a[2]), out_type = (int)whole(a[3]), kind = (int)whole(a[4]), wide = (int)whole(a[7]);
    const double max_norm = number(a[5]), eps = number(a[6]);
    const auto gpu = (c10::DeviceIndex)whole(a[8]);
    const at::Tensor result = at::detail::empty_cuda({2}, wide == FO_F64 ? at::kDouble : at::kFloat, c10::Device(c10::kCUDA, gpu),
                                                     c10::nullopt);
    const OnGpu on(gpu);
    const cudaStream_t st = c10::cuda::getCurrentCUDAStream(gpu).stream();
    const at::Tensor ws = workspace(gpu, st, fused_grad_workspace_bytes());
    if (clip)
        check_status(fused_grad_clip(list, count, in_type, out_type, kind, max_norm, eps, result.data_ptr(), wide, ws.data_ptr(),
                                     (size_t)ws.numel(), st), "fused_grad_clip");
    else
        check_status(fused_grad_norm(list, count, in_type, kind, max_norm, eps, result.data_ptr(), wide, ws.data_ptr(),
                                     (size_t)ws.numel(), st), "fused_grad_norm");
    return THPVariable_Wrap(result);
}

// adamw(list, grad_type, weight_type, lr, beta1, beta2, eps, step, factor, gpu)
PyObject *adamw_impl(PyObject *const *a)
{
    int count;
    const fo_adam_tensor *list = packed_list<fo_adam_tensor>(a[0], &count);
    const int grad_type = (int)whole(a[1]), weight_type = (int)whole(a[2]);
    const at::Tensor *factor = tensor_of(a[8], "factor");
    const auto gpu = (c10::DeviceIndex)whole(a[9]);
    if (factor)
        require(factor->numel() == 1 && factor->is_cuda() && factor->get_device() == gpu
                    && (factor->scalar_type() == at::kFloat || factor->scalar_type() == at::kDouble),
                "factor is not one float on the gradients' device");
    const OnGpu on(gpu);
    check_status(fused_adamw(list, count, grad_type, weight_type, number(a[3]), number(a[4]), number(a[5]), number(a[6]),
                             whole(a[7]), factor ? factor->data_ptr() : nullptr,
                             factor ? type_code(factor->scalar_type()) : FO_F32,
                             c10::cuda::getCurrentCUDAStream(gpu).stream()), "fused_adamw");
    Py_RETURN_NONE;
}

template <PyObject *(*IMPL)(PyObject *const *), int N>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments are needed", N);
        return nullptr;
    }
    try {
        return IMPL(args);
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Raised &) {
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}
template <PyObject *(*IMPL)(PyObject *const *), int N>
PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<IMPL, N>)), METH_FASTCALL, nullptr};
}

PyObject *connect(PyObject *, PyObject *args)
{
    PyObject *error, *ws;
    if (!PyArg_ParseTuple(args, "OO", &error, &ws)) return nullptr;
    Py_INCREF(error), Py_INCREF(ws);
    Py_XDECREF(g_error), Py_XDECREF(g_workspace);
    g_error = error, g_workspace = ws;
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {method<block_norm_impl, 11>("block_norm"), method<block_norm_grad_impl, 11>("block_norm_grad"),
                           method<grad_norm_impl, 9>("grad_norm"), method<adamw_impl, 10>("adamw"),
                           {"connect", connect, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_training", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__training() { return PyModule_Create(&g_module); }
