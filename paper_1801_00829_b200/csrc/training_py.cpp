// CPython extension behind training.py: argument checks and marshalling of calls that are made once per layer or step and
// for small inputs take less time on the GPU than a call assembled in Python takes on the host (block norm 15 us, its
// gradient 30; here 5 and 11), and of lists whose tensors are looked at in every call (7 to 9 ns each).  Nothing
// here computes.
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <map>
#include <string>
#include <utility>
#include <vector>

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

at::ScalarType dtype_of(PyObject *o, const char *name)
{
    if (!THPDtype_Check(o)) throw Refused(std::string(name) + " is not a dtype");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

// The address of a tensor of which `reach` elements from its first one on are used; its storage may have been resized.
void *data_of(const at::Tensor &t, int64_t reach, const char *name)
{
    if (reach <= 0) return nullptr;
    const c10::TensorImpl &impl = *t.unsafeGetTensorImpl();
    c10::StorageImpl &held = *impl.storage().unsafeGetStorageImpl();
    const size_t bytes = impl.dtype().itemsize(), at_byte = (size_t)impl.storage_offset() * bytes;
    if (held.nbytes() < at_byte + (size_t)reach * bytes)
        throw Refused(std::string(name) + ": the tensor's storage is smaller than the tensor");
    return static_cast<char *>(held.mutable_data()) + at_byte;
}

// The operators record no graph: a tensor that autograd follows would lose its gradient without a word.
void outside_graph(const at::Tensor &t, const char *name)
{
    if (t.requires_grad() && c10::GradMode::is_enabled())
        throw Refused(std::string(name) + " requires a gradient, and this call records none: call it under torch.no_grad(), or in an "
                                          "autograd.Function whose backward is fused_block_norm_grad");
}
// `t` was written: what autograd saved of it is no longer what it was.
void written(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
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
        outside_graph(*t, name);
        if (cols > 1 && t->stride(1) != 1) throw Refused(std::string("rows of ") + name + " must be contiguous");
        *ld = t->stride(0);
        if (*ld < cols) {
            if (rows > 1) throw Refused(std::string("rows of ") + name + " overlap");
            *ld = cols;
        }
        return data_of(*t, cols > 0 ? (rows - 1) * *ld + cols : 0, name);
    }
    void *vector(const at::Tensor *t, at::ScalarType type, const char *name) const
    {
        if (!t) return nullptr;
        if (t->dim() != 1 || t->size(0) != cols || t->scalar_type() != type || !t->is_cuda() || t->get_device() != gpu
            || !t->is_contiguous())
            refuse(*t, name, "a contiguous vector over the columns", type);
        outside_graph(*t, name);
        return data_of(*t, cols, name);
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
        outside_graph(*t, "gate");
        ld = n > 1 ? t->stride(along) : 1;
        require(access == FO_AT_ROW ? ld >= 1 : ld == 1, "stride of the gate");
        p = data_of(*t, (n - 1) * ld + 1, "gate");
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

// block_norm(x, f, post, gate, scale, col_scale, pre, out_h, out_y, stats, block_type, stream_type)
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
    at::ScalarType stream = x || !out_h ? first.scalar_type() : out_h->scalar_type();
    if (a[11] != Py_None) {
        const at::ScalarType wanted = dtype_of(a[11], "stream_type");
        require((!x && !out_h) || wanted == stream, "stream_type is not the type of x and out_h");
        stream = wanted;
    }
    at::ScalarType block = f ? f->scalar_type() : out_y ? out_y->scalar_type() : stream;
    if (!f) {
        require(!post.given() && !gate.t && !col_scale, "post, gate and col_scale need a block output f");
        if (a[10] != Py_None) {
            block = dtype_of(a[10], "block_type");
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
    if (out_h) written(*out_h);
    if (out_y) written(*out_y);
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

at::Tensor new_workspace(c10::DeviceIndex gpu, size_t bytes)
{
    PyObject *o = PyObject_CallFunction(g_workspace, "in", (int)gpu, (Py_ssize_t)bytes);
    if (!o) throw Raised();
    const at::Tensor t = THPVariable_Unpack(o);
    Py_DECREF(o);
    return t;
}
// The stream's scratch; a call that is captured into a graph gets one of its own (binding.workspace).
at::Tensor workspace(c10::DeviceIndex gpu, cudaStream_t stream, size_t bytes)
{
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone)
        return new_workspace(gpu, bytes);
    static auto *cache = new std::map<std::pair<int, cudaStream_t>, at::Tensor>();      // outlives the interpreter
    at::Tensor &buf = (*cache)[{gpu, stream}];
    if (!buf.defined() || (size_t)buf.numel() < bytes) buf = new_workspace(gpu, bytes);
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
    const at::ScalarType block = f ? f->scalar_type() : dy ? dy->scalar_type()      // else as in the forward call
                                 : stream == at::kFloat ? vector_type(stream, post, pre, col_scale) : stream;
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
        outside_graph(*stats, "stats");
        n.stats = data_of(*stats, 4 * call.rows, "stats");
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

// What the tensors of one list are: their type, on one GPU.
struct Kind {
    at::ScalarType type;
    c10::DeviceIndex gpu;
};

// One Python list of tensors that belongs to a call.  Tensors can change under a list that is kept: `t.data = other` or a
// storage that is resized moves them, to another size or type at that.  So every call looks at every tensor again, and
// nothing of an earlier call is used.  That takes 7 to 9 ns a tensor on the host, for what it reads of each; comparing with
// what an earlier call saw took as long.
class Tensors {
    PyObject *list_;
    const char *name_;

    [[noreturn]] void refuse(const char *what) const { throw Refused(std::string(name_) + ": " + what); }

public:
    Tensors(PyObject *list, const char *name) : list_(list), name_(name)
    {
        require(PyList_Check(list), "tensors are given as a list");
    }
    size_t count() const { return (size_t)PyList_GET_SIZE(list_); }
    bool is(PyObject *list) const { return list == list_; }
    const at::Tensor &at(size_t k) const
    {
        PyObject *o = PyList_GET_ITEM(list_, (Py_ssize_t)k);
        if (!THPVariable_Check(o)) refuse("not a tensor");
        return THPVariable_Unpack(o);
    }
    void same_count(size_t n) const
    {
        if (count() != n) throw Refused(std::string(name_) + ": " + std::to_string(count()) + " tensors for " + std::to_string(n));
    }
    // put(k, address of tensor k's elements), of which there have to be n(k); `write`: the call will write them
    template <class Size, class Put>
    void read(const Kind &kind, bool write, Size n, Put put) const
    {
        const caffe2::TypeMeta type = c10::scalarTypeToTypeMeta(kind.type);
        const c10::Device device(c10::kCUDA, kind.gpu);
        const size_t bytes = type.itemsize(), many = count();
        PyTypeObject *known = nullptr;                       // the Python type of the tensor before
        c10::StorageImpl *one = nullptr;                     // its storage: neighbours in a bucket share it
        char *begin = nullptr;
        size_t held = 0;
        for (size_t k = 0; k < many; ++k) {
            PyObject *o = PyList_GET_ITEM(list_, (Py_ssize_t)k);
            if (Py_TYPE(o) != known) at(k), known = Py_TYPE(o);
            const c10::TensorImpl &t = *THPVariable_Unpack(o).unsafeGetTensorImpl();
            if (t.dtype() != type || t.device() != device) refuse("tensors of one type on one device are needed");
            if (!t.is_contiguous()) refuse("tensors must be contiguous");
            const int64_t want = n(k, t);
            if (t.numel() != want) refuse("sizes differ");
            c10::StorageImpl *const storage = t.storage().unsafeGetStorageImpl();
            if (storage != one) one = storage, begin = static_cast<char *>(storage->mutable_data()), held = storage->nbytes();
            const size_t at_byte = (size_t)t.storage_offset() * bytes;
            if (want && held < at_byte + (size_t)want * bytes) refuse("a tensor's storage is smaller than the tensor");
            put(k, want ? begin + at_byte : nullptr);
            if (write) written(THPVariable_Unpack(o));
        }
    }
};

// The kind of a list's first tensor.
Kind kind_of(const Tensors &grads)
{
    if (grads.count() == 0) return {at::kFloat, -1};
    const at::Tensor &t = grads.at(0);
    require(t.is_cuda(), "fused operators need CUDA tensors (no CPU path)");
    type_code(t.scalar_type());
    return {t.scalar_type(), t.get_device()};
}

bool sixteen_bits(at::ScalarType t) { return t == at::kBFloat16 || t == at::kHalf; }

// Gradients, and the tensors their clipped values go to (None: not wanted; the list itself: in place).
struct GradTensors {
    std::vector<fo_tensor> c;
    Kind kind;
    at::ScalarType out_type;

    GradTensors(PyObject *grads, PyObject *outs, bool write)
    {
        const Tensors in(grads, "grads");
        kind = kind_of(in), out_type = kind.type;
        c.resize(in.count());
        in.read(kind, write && in.is(outs), [&](size_t k, const c10::TensorImpl &t) { return c[k].n = t.numel(); },
                [&](size_t k, void *p) { c[k].in = c[k].out = p; });
        if (outs == Py_None || in.is(outs)) return;
        const Tensors out(outs, "outs");
        out.same_count(c.size());
        if (c.empty()) return;
        out_type = out.at(0).scalar_type();
        if (out_type != kind.type && !(sixteen_bits(kind.type) && out_type == at::kFloat))
            throw Refused(std::string("clipped values of ") + c10::toString(out_type) + " from gradients of "
                          + c10::toString(kind.type));
        out.read({out_type, kind.gpu}, write, [&](size_t k, const c10::TensorImpl &) { return c[k].n; },
                 [&](size_t k, void *p) { c[k].out = p; });
    }
};

// The lists of an AdamW update: params, grads, m, v, the new params, m and v, weights (or None), decay (doubles, packed).
struct AdamTensors {
    std::vector<fo_adam_tensor> c;
    Kind kind;
    at::ScalarType weight_type = at::kBFloat16;

    AdamTensors(PyObject *const *a, bool write)
    {
        const Tensors grads(a[1], "grads");
        kind = kind_of(grads);
        c.resize(grads.count());
        require(PyBytes_Check(a[8]) && (size_t)PyBytes_GET_SIZE(a[8]) == c.size() * sizeof(double),
                "decay: one value per tensor is needed");
        grads.read(kind, false, [&](size_t k, const c10::TensorImpl &t) { return c[k].n = t.numel(); }, [&](size_t k, void *p) {
            c[k].g = p;
            memcpy(&c[k].decay, PyBytes_AS_STRING(a[8]) + k * sizeof(double), sizeof(double));
        });
        const Kind wide = {kind.type == at::kDouble ? at::kDouble : at::kFloat, kind.gpu};
        // the new values: every list may be the one it comes from
        const auto both = [&](PyObject *in, const char *in_name, PyObject *out, const char *out_name, const void *fo_adam_tensor::*p,
                              void *fo_adam_tensor::*q) {
            take(in, in_name, wide, write && out == in, [&](size_t k, void *v) { c[k].*p = c[k].*q = v; });
            if (out != in) take(out, out_name, wide, write, [&](size_t k, void *v) { c[k].*q = v; });
        };
        both(a[0], "params", a[4], "params out", &fo_adam_tensor::p, &fo_adam_tensor::p_out);
        both(a[2], "m", a[5], "m out", &fo_adam_tensor::m, &fo_adam_tensor::m_out);
        both(a[3], "v", a[6], "v out", &fo_adam_tensor::v, &fo_adam_tensor::v_out);
        if (a[7] == Py_None || c.empty()) return;
        const Tensors weights(a[7], "weights");
        weights.same_count(c.size());
        weight_type = weights.at(0).scalar_type();
        require(sixteen_bits(weight_type), "weights are bfloat16 or float16");
        require(kind.type != at::kDouble, "no 16-bit weights beside gradients of float64");
        take(a[7], "weights", {weight_type, kind.gpu}, write, [&](size_t k, void *p) { c[k].weights = p; });
    }

private:
    template <class Put>
    void take(PyObject *list, const char *name, const Kind &of, bool write, Put put)
    {
        const Tensors ts(list, name);
        ts.same_count(c.size());
        ts.read(of, write, [&](size_t k, const c10::TensorImpl &) { return c[k].n; }, put);
    }
};

// check_grads(grads, outs), check_adam(the nine of AdamTensors): refuse what a call would refuse
PyObject *check_grads_impl(PyObject *const *a)
{
    GradTensors(a[0], a[1], false);
    Py_RETURN_NONE;
}
PyObject *check_adam_impl(PyObject *const *a)
{
    AdamTensors(a, false);
    Py_RETURN_NONE;
}

// grad_norm(grads, outs or None: no clipping, norm_kind, max_norm, eps, result_type, gpu of an empty list) -> (norm, factor)
PyObject *grad_norm_impl(PyObject *const *a)
{
    const GradTensors t(a[0], a[1], true);
    const bool clip = a[1] != Py_None;
    const int kind = (int)whole(a[2]), wide = (int)whole(a[5]), count = (int)t.c.size();
    const double max_norm = number(a[3]), eps = number(a[4]);
    const auto gpu = t.kind.gpu >= 0 ? t.kind.gpu : (c10::DeviceIndex)whole(a[6]);
    const at::Tensor result = at::detail::empty_cuda({2}, wide == FO_F64 ? at::kDouble : at::kFloat, c10::Device(c10::kCUDA, gpu),
                                                     c10::nullopt);
    const OnGpu on(gpu);
    const cudaStream_t st = c10::cuda::getCurrentCUDAStream(gpu).stream();
    const at::Tensor ws = workspace(gpu, st, fused_grad_workspace_bytes());
    if (clip)
        check_status(fused_grad_clip(t.c.data(), count, type_code(t.kind.type), type_code(t.out_type), kind, max_norm, eps,
                                     result.data_ptr(), wide, ws.data_ptr(), (size_t)ws.numel(), st), "fused_grad_clip");
    else
        check_status(fused_grad_norm(t.c.data(), count, type_code(t.kind.type), kind, max_norm, eps, result.data_ptr(), wide,
                                     ws.data_ptr(), (size_t)ws.numel(), st), "fused_grad_norm");
    return THPVariable_Wrap(result);
}

// adamw(the nine of AdamTensors, lr, beta1, beta2, eps, step, factor)
PyObject *adamw_impl(PyObject *const *a)
{
    const AdamTensors t(a, true);
    const at::Tensor *factor = tensor_of(a[14], "factor");
    const c10::DeviceIndex gpu = t.kind.gpu;
    if (factor)
        require(factor->numel() == 1 && factor->is_cuda() && factor->get_device() == gpu
                    && (factor->scalar_type() == at::kFloat || factor->scalar_type() == at::kDouble),
                "factor is not one float on the gradients' device");
    const OnGpu on(gpu);
    check_status(fused_adamw(t.c.data(), (int)t.c.size(), type_code(t.kind.type), type_code(t.weight_type), number(a[9]), number(a[10]),
                             number(a[11]), number(a[12]), whole(a[13]), factor ? data_of(*factor, 1, "factor") : nullptr,
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

PyMethodDef g_methods[] = {method<block_norm_impl, 12>("block_norm"), method<block_norm_grad_impl, 11>("block_norm_grad"),
                           method<grad_norm_impl, 7>("grad_norm"), method<adamw_impl, 15>("adamw"),
                           method<check_grads_impl, 2>("check_grads"), method<check_adam_impl, 9>("check_adam"),
                           {"connect", connect, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_training", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__training() { return PyModule_Create(&g_module); }
