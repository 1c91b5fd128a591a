// Argument checks and marshalling of lm.py's calls, in the CPython extension beside those of training.py: a call takes 4 to 6 us
// on the host, which is most of what a decoding step of these operators costs.  Nothing here computes.
#include "training_py.h"
#include "lm_py.h"

#include <algorithm>

namespace fo_py {
namespace {

[[noreturn]] void refuse(const std::string &name, const std::string &needed, const at::Tensor &t)
{
    std::string s = name + ": " + needed + " is needed, not " + c10::toString(t.scalar_type()) + " [";
    for (int64_t n : t.sizes()) s += " " + std::to_string(n);
    throw Refused(s + " ] on " + t.device().str());
}
[[noreturn]] void refuse(const char *name, const char *what) { throw Refused(std::string(name) + what); }

at::ScalarType wide_type(at::ScalarType t) { return t == at::kDouble ? at::kDouble : at::kFloat; }
bool sixteen(at::ScalarType t) { return t == at::kBFloat16 || t == at::kHalf; }

c10::DeviceIndex gpu_of(const at::Tensor &t)
{
    require(t.is_cuda(), "fused operators need CUDA tensors (no CPU path)");
    return t.get_device();
}
bool on_gpu(const at::Tensor &t, c10::DeviceIndex gpu) { return t.is_cuda() && t.get_device() == gpu; }

at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, c10::DeviceIndex gpu)
{
    return at::detail::empty_cuda(sizes, type, c10::Device(c10::kCUDA, gpu), c10::nullopt);
}

// The address of a tensor, all of whose elements are in its storage.
void *all_of(const at::Tensor &t, const char *name)
{
    int64_t reach = 1;
    for (int64_t d = 0; d < t.dim(); ++d) {
        if (t.size(d) == 0) return nullptr;
        reach += (t.size(d) - 1) * t.stride(d);
    }
    return data_of(t, reach, name);
}

// No two elements of a tensor that is written share a place.
void distinct(const at::Tensor &t, const char *name)
{
    int order[4], n = 0;
    for (int d = 0; d < (int)t.dim(); ++d) {
        if (t.size(d) == 0) return;
        if (t.size(d) > 1) order[n++] = d;
    }
    std::sort(order, order + n, [&](int a, int b) { return t.stride(a) < t.stride(b); });
    int64_t extent = 1;
    for (int k = 0; k < n; ++k) {
        if (t.stride(order[k]) < extent) refuse(name, ": elements that share a place cannot be written");
        extent += (t.size(order[k]) - 1) * t.stride(order[k]);
    }
}

// A tensor of the given sizes, whose neighbours along the last dimension are neighbours in memory.
void *rows_of(const at::Tensor *t, at::IntArrayRef sizes, at::ScalarType type, c10::DeviceIndex gpu, const char *name,
              bool write = false)
{
    if (!t) return nullptr;
    if (t->sizes() != sizes || t->scalar_type() != type || !on_gpu(*t, gpu)) {
        std::string s = std::string(c10::toString(type)) + " [";
        for (int64_t n : sizes) s += " " + std::to_string(n);
        refuse(name, s + " ] on GPU " + std::to_string((int)gpu), *t);
    }
    outside_graph(*t, name);
    if (t->dim() > 0 && sizes.back() > 1 && t->stride(-1) != 1) refuse(name, ": neighbours along the last dimension must be neighbours in memory");
    if (write) distinct(*t, name);
    return all_of(*t, name);
}
void *packed_of(const at::Tensor *t, at::IntArrayRef sizes, at::ScalarType type, c10::DeviceIndex gpu, const char *name,
                bool write = false)
{
    void *p = rows_of(t, sizes, type, gpu, name, write);
    if (t && !t->is_contiguous()) refuse(name, " must be contiguous");
    return p;
}
int int_code(const at::Tensor &t, const char *name)
{
    if (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) refuse(name, ": int32 or int64 is needed");
    return t.scalar_type() == at::kLong ? FO_I64 : FO_I32;
}

PyObject *given_or_new(PyObject *given, const at::Tensor &t)
{
    if (given != Py_None) return Py_INCREF(given), given;
    return or_none(t);
}
PyObject *pair_of(PyObject *a, PyObject *b)
{
    PyObject *out = a && b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a), Py_XDECREF(b);
    return out;
}

// A dict of results that is being filled.
struct Results {
    PyObject *dict = PyDict_New();
    Results()
    {
        if (!dict) throw Raised();
    }
    ~Results() { Py_XDECREF(dict); }
    Results(const Results &) = delete;
    void put(const char *name, PyObject *o)
    {
        const int rc = o ? PyDict_SetItemString(dict, name, o) : -1;
        Py_XDECREF(o);
        if (rc != 0) throw Raised();
    }
    PyObject *release()
    {
        PyObject *d = dict;
        dict = nullptr;
        return d;
    }
};

cudaStream_t stream_of(c10::DeviceIndex gpu) { return c10::cuda::getCurrentCUDAStream(gpu).stream(); }

// ------------------------------------------------------------------------------------------------------------ head norms
// Sizes and strides of a tensor of heads: (tokens, heads, dim) or (batch, tokens, heads, dim).
struct Heads {
    int64_t batch = 1, tokens, heads, dim;
    fo_strides at = {0, 0, 0};
    explicit Heads(const at::Tensor &t, const char *name)
    {
        const int64_t n = t.dim();
        if (n != 3 && n != 4) refuse(name, ": (tokens, heads, dim) or (batch, tokens, heads, dim) is needed");
        if (n == 4) batch = t.size(0), at.batch = t.stride(0);
        tokens = t.size(n - 3), heads = t.size(n - 2), dim = t.size(n - 1);
        at.token = t.stride(n - 3), at.head = t.stride(n - 2);
    }
};

struct HeadNormArg {
    const at::Tensor *weight = nullptr, *bias = nullptr;
    fo_norm c = {};
    HeadNormArg(PyObject *o, const char *name)
    {
        if (o == Py_None) return;
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) refuse(name, " is (kind, weight, bias, eps)");
        PyObject *kind = PyTuple_GET_ITEM(o, 0);
        c.kind = is(kind, "rms") ? FO_NORM_RMS : is(kind, "layer") ? FO_NORM_LAYER : FO_NORM_NONE;
        if (c.kind == FO_NORM_NONE) refuse(name, ": a norm is \"rms\" or \"layer\"");
        weight = tensor_of(PyTuple_GET_ITEM(o, 1), "weight");
        bias = tensor_of(PyTuple_GET_ITEM(o, 2), "bias");
        c.eps = number(PyTuple_GET_ITEM(o, 3));
    }
    // the type of its vectors, or `none`
    at::ScalarType type(at::ScalarType none) const { return weight ? weight->scalar_type() : bias ? bias->scalar_type() : none; }
    void check(int64_t dim, at::ScalarType vec, c10::DeviceIndex gpu)
    {
        c.weight = packed_of(weight, {dim}, vec, gpu, "weight");
        c.bias = packed_of(bias, {dim}, vec, gpu, "bias");
    }
};

// (cos, sin, positions, pairing, sections) or None
fo_rotation rotation_of(PyObject *o, const Heads &like, bool batched, at::ScalarType type, c10::DeviceIndex gpu)
{
    fo_rotation r = {};
    if (o == Py_None) return r;
    require(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 5, "a rotation is (cos, sin, positions, pairing, sections)");
    const at::Tensor *cos = tensor_of(PyTuple_GET_ITEM(o, 0), "cos"), *sin = tensor_of(PyTuple_GET_ITEM(o, 1), "sin");
    const at::Tensor *pos = tensor_of(PyTuple_GET_ITEM(o, 2), "positions");
    PyObject *how = PyTuple_GET_ITEM(o, 3), *sections = PyTuple_GET_ITEM(o, 4);
    require(cos && sin && pos, "a rotation needs cos, sin and positions");
    require(cos->dim() == 2, "cos and sin are (positions, pairs)");
    r.rows = cos->size(0);
    require(2 * cos->size(1) <= like.dim, "more pairs than the heads have");
    r.pairs = (int32_t)cos->size(1);
    r.pairing = is(how, "halves") ? FO_PAIR_HALVES : is(how, "neighbours") || is(how, "pairs") ? FO_PAIR_NEIGHBOURS : -1;
    require(r.pairing >= 0, "a rotation's pairing is \"halves\" or \"pairs\"");
    r.cos_table = rows_of(cos, cos->sizes(), wide_type(type), gpu, "cos");
    r.sin_table = rows_of(sin, cos->sizes(), wide_type(type), gpu, "sin");
    r.ld_cos = r.rows > 1 ? cos->stride(0) : r.pairs, r.ld_sin = r.rows > 1 ? sin->stride(0) : r.pairs;
    require(r.ld_cos >= r.pairs && r.ld_sin >= r.pairs, "rows of cos or sin overlap");
    r.axes = 1, r.section[0] = r.pairs;
    if (sections != Py_None) {
        require(PyTuple_Check(sections) && PyTuple_GET_SIZE(sections) >= 1 && PyTuple_GET_SIZE(sections) <= FO_MAX_AXES,
                "sections are a tuple of one to four numbers of pairs");
        r.axes = (int32_t)PyTuple_GET_SIZE(sections);
        int64_t sum = 0;
        for (int k = 0; k < r.axes; ++k) {
            const long long n = whole(PyTuple_GET_ITEM(sections, k));
            require(n >= 0 && n <= r.pairs, "a section is a number of pairs");
            r.section[k] = (int32_t)n, sum += n;
        }
        require(sum == r.pairs, "the sections' pairs are not the table's");
    }
    // positions: ([axes,] [batch,] tokens); without the batch they are those of every sequence
    const int lead = sections != Py_None;
    r.position_type = int_code(*pos, "positions");
    const bool each = batched && pos->dim() == lead + 2;
    if (!on_gpu(*pos, gpu) || pos->dim() != lead + 1 + each || (lead && pos->size(0) != r.axes) || (each && pos->size(lead) != like.batch)
        || pos->size(-1) != like.tokens)
        refuse("positions", lead ? "(axes, batch, tokens) or (axes, tokens)" : "(batch, tokens) or (tokens)", *pos);
    r.positions = all_of(*pos, "positions");
    r.position_axis = lead ? pos->stride(0) : 0, r.position_batch = each ? pos->stride(lead) : 0, r.position_token = pos->stride(-1);
    return r;
}

at::ScalarType vectors_of(at::ScalarType type, const HeadNormArg &a, const HeadNormArg &b)
{
    const at::ScalarType vec = a.type(b.type(type));
    require(vec == type || (vec == at::kFloat && sixteen(type)), "weights and biases have the heads' type, or float32 beside 16 bits");
    return vec;
}

// A second tensor of heads agrees with the first.
void same_tokens(const Heads &a, const Heads &b, const at::Tensor &ta, const at::Tensor &tb, const char *name)
{
    if (a.batch != b.batch || a.tokens != b.tokens || a.dim != b.dim || ta.scalar_type() != tb.scalar_type() || ta.dim() != tb.dim()
        || !on_gpu(tb, ta.get_device()))
        refuse(name, ": batch, tokens, dim, type or GPU differ from the other heads'");
}

}  // namespace

// head_norm(q, k, q_norm, k_norm, rotate, out_q, out_k)
PyObject *head_norm_impl(PyObject *const *a)
{
    static const char *const names[2] = {"q", "k"}, *const outs[2] = {"out_q", "out_k"}, *const norms[2] = {"q_norm", "k_norm"};
    const at::Tensor *x[2] = {tensor_of(a[0], "q"), tensor_of(a[1], "k")}, *out[2] = {tensor_of(a[5], "out_q"), tensor_of(a[6], "out_k")};
    require(x[0], "q is needed");
    require(x[1] || (a[3] == Py_None && !out[1]), "k_norm and out_k need k");
    const c10::DeviceIndex gpu = gpu_of(*x[0]);
    const at::ScalarType type = x[0]->scalar_type();
    const Heads first(*x[0], "q");
    HeadNormArg norm[2] = {{a[2], norms[0]}, {a[3], norms[1]}};
    const at::ScalarType vec = vectors_of(type, norm[0], norm[1]);
    fo_head_norm n = {};
    n.batch = first.batch, n.tokens = first.tokens, n.type = type_code(type), n.vec_type = type_code(vec);
    require(first.dim <= FO_HEAD_MAX_DIM, "heads of at most 512 values");
    n.dim = (int32_t)first.dim, n.count = x[1] ? 2 : 1;
    n.rotation = rotation_of(a[4], first, x[0]->dim() == 4, type, gpu);
    at::Tensor made[2];
    for (int k = 0; k < n.count; ++k) {
        const Heads h(*x[k], names[k]);
        if (k) same_tokens(first, h, *x[0], *x[1], "k");
        fo_heads &t = n.t[k];
        norm[k].check(first.dim, vec, gpu);
        t.heads = h.heads, t.norm = norm[k].c, t.x_at = h.at;
        t.x = rows_of(x[k], x[k]->sizes(), type, gpu, names[k]);
        if (!out[k]) made[k] = make(x[k]->sizes(), type, gpu);
        const at::Tensor &to = out[k] ? *out[k] : made[k];
        t.y = rows_of(&to, x[k]->sizes(), type, gpu, outs[k], out[k] != nullptr);
        t.y_at = Heads(to, outs[k]).at;
    }
    const OnGpu on(gpu);
    check_status(fused_head_norm(&n, stream_of(gpu)), "fused_head_norm");
    for (int k = 0; k < 2; ++k)
        if (out[k]) written(*out[k]);
    PyObject *q = given_or_new(a[5], made[0]);
    return pair_of(q, given_or_new(a[6], made[1]));
}

// head_norm_grad(dq, dk, q, k, q_norm, k_norm, rotate, out_q, out_k)
PyObject *head_norm_grad_impl(PyObject *const *a)
{
    static const char *const names[2] = {"q", "k"}, *const grads[2] = {"dq", "dk"}, *const outs[2] = {"out_q", "out_k"},
                      *const norms[2] = {"q_norm", "k_norm"}, *const ws_names[2] = {"q_w", "k_w"}, *const bs_names[2] = {"q_b", "k_b"};
    const at::Tensor *dy[2] = {tensor_of(a[0], "dq"), tensor_of(a[1], "dk")}, *x[2] = {tensor_of(a[2], "q"), tensor_of(a[3], "k")};
    const at::Tensor *out[2] = {tensor_of(a[7], "out_q"), tensor_of(a[8], "out_k")};
    require(dy[0] || dy[1], "dq or dk is needed");
    const at::Tensor &like = dy[0] ? *dy[0] : *dy[1];
    const c10::DeviceIndex gpu = gpu_of(like);
    const at::ScalarType type = like.scalar_type();
    const Heads first(like, dy[0] ? "dq" : "dk");
    HeadNormArg norm[2] = {{dy[0] ? a[4] : Py_None, norms[0]}, {dy[1] ? a[5] : Py_None, norms[1]}};
    const at::ScalarType vec = vectors_of(type, norm[0], norm[1]), sums = wide_type(type);
    fo_head_norm_grad n = {};
    n.batch = first.batch, n.tokens = first.tokens, n.type = type_code(type), n.vec_type = type_code(vec);
    require(first.dim <= FO_HEAD_MAX_DIM, "heads of at most 512 values");
    n.dim = (int32_t)first.dim;
    n.rotation = rotation_of(a[6], first, like.dim() == 4, type, gpu);
    Results got;
    bool summed = false;
    for (int k = 0; k < 2; ++k) {
        if (!dy[k]) {
            if (out[k]) refuse(outs[k], " without its gradient");
            continue;
        }
        const Heads h(*dy[k], grads[k]);
        same_tokens(first, h, like, *dy[k], grads[k]);
        fo_heads_grad &t = n.t[n.count++];
        norm[k].check(first.dim, vec, gpu);
        t.heads = h.heads, t.norm = norm[k].c, t.dy_at = h.at;
        t.dy = rows_of(dy[k], dy[k]->sizes(), type, gpu, grads[k]);
        if (t.norm.kind != FO_NORM_NONE) {
            if (!x[k]) refuse(names[k], " is needed with a norm");
            t.x = rows_of(x[k], dy[k]->sizes(), type, gpu, names[k]);
            t.x_at = Heads(*x[k], names[k]).at;
        }
        at::Tensor made;
        if (!out[k]) made = make(dy[k]->sizes(), type, gpu);
        const at::Tensor &to = out[k] ? *out[k] : made;
        t.dx = rows_of(&to, dy[k]->sizes(), type, gpu, outs[k], out[k] != nullptr);
        t.dx_at = Heads(to, outs[k]).at;
        got.put(names[k], given_or_new(a[7 + k], made));
        const auto sum = [&](const at::Tensor *of, const char *name) -> void * {
            if (!of) return nullptr;
            const at::Tensor s = make({first.dim}, sums, gpu);
            got.put(name, or_none(s));
            summed = true;
            return s.data_ptr();
        };
        t.dweight = sum(norm[k].weight, ws_names[k]);
        t.dbias = sum(norm[k].bias, bs_names[k]);
    }
    const OnGpu on(gpu);
    const cudaStream_t st = stream_of(gpu);
    at::Tensor ws;
    if (summed) ws = workspace(gpu, st, fused_head_norm_grad_workspace_bytes(n.dim, n.type));
    check_status(fused_head_norm_grad(&n, summed ? ws.data_ptr() : nullptr, summed ? (size_t)ws.numel() : 0, st), "fused_head_norm_grad");
    for (int k = 0; k < 2; ++k)
        if (out[k]) written(*out[k]);
    return got.release();
}

// ------------------------------------------------------------------------------------------------------------ recurrence
namespace {

// What forward and gradient have in common: (batch, tokens, channels), or (tokens, channels) as a batch of one.
struct ScanArgs {
    int64_t batch = 1, tokens, channels;
    c10::DeviceIndex gpu;
    at::ScalarType type, gate_type, wide;
    std::vector<int64_t> state_sizes;
    int decay, mix;
    const at::Tensor &like;

    ScanArgs(const at::Tensor &x, const at::Tensor *gate, PyObject *decay_name, PyObject *mix_name)
        : gpu(gpu_of(x)), type(x.scalar_type()), wide(wide_type(x.scalar_type())), like(x)
    {
        const int64_t n = x.dim();
        require(n == 2 || n == 3, "(batch, tokens, channels) or (tokens, channels) is needed");
        if (n == 3) batch = x.size(0), state_sizes.push_back(batch);
        tokens = x.size(n - 2), channels = x.size(n - 1);
        state_sizes.push_back(channels);
        require(gate, "the gate is needed");
        gate_type = gate->scalar_type();
        require(gate_type == type || (gate_type == at::kFloat && sixteen(type)), "the gate has the type of x, or float32 beside 16 bits");
        decay = is(decay_name, "value") ? FO_DECAY_VALUE : is(decay_name, "sigmoid") ? FO_DECAY_SIGMOID : is(decay_name, "exp") ? FO_DECAY_EXP : -1;
        mix = is(mix_name, "one") ? FO_MIX_ONE : is(mix_name, "rest") ? FO_MIX_REST : is(mix_name, "root") ? FO_MIX_ROOT : -1;
        require(decay >= 0, "a decay is \"value\", \"sigmoid\" or \"exp\"");
        require(mix >= 0, "a mix is \"one\", \"rest\" or \"root\"");
        type_code(type);
    }
    void *rows(const at::Tensor *t, at::ScalarType of, const char *name, fo_rows *at, bool write = false) const
    {
        void *p = rows_of(t, like.sizes(), of, gpu, name, write);
        if (t) *at = {t->dim() == 3 ? t->stride(0) : 0, t->stride(-2)};
        return p;
    }
    void *state(const at::Tensor *t, const char *name, bool write = false) const { return packed_of(t, state_sizes, wide, gpu, name, write); }
    void *marks(const at::Tensor *t, fo_rows *at) const
    {
        if (!t) return nullptr;
        if ((t->scalar_type() != at::kBool && t->scalar_type() != at::kByte) || t->sizes() != like.sizes().slice(0, like.dim() - 1) || !on_gpu(*t, gpu))
            refuse("reset", "bool or uint8 (batch, tokens)", *t);
        *at = {t->dim() == 2 ? t->stride(0) : 0, t->stride(-1)};
        return all_of(*t, "reset");
    }
    void *ends(const at::Tensor *t, int32_t *code) const
    {
        if (!t) return nullptr;
        *code = int_code(*t, "lengths");
        if (t->numel() != batch || t->dim() > 1 || !t->is_contiguous() || !on_gpu(*t, gpu)) refuse("lengths", "a contiguous vector over the batch", *t);
        return all_of(*t, "lengths");
    }
};

// Long sequences take scratch; a decoding step that is captured into a graph takes none, and so the graph clears none.
struct ScanScratch {
    at::Tensor held;
    void *at = nullptr;
    size_t bytes;
    ScanScratch(const ScanArgs &c, cudaStream_t st) : bytes(fused_scan_workspace_bytes(c.tokens))
    {
        if (bytes) held = workspace(c.gpu, st, bytes), at = held.data_ptr(), bytes = (size_t)held.numel();
    }
};

}  // namespace

// scan(x, gate, decay, mix, state, reset, lengths, out, out_state)
PyObject *scan_impl(PyObject *const *a)
{
    const at::Tensor *x = tensor_of(a[0], "x"), *gate = tensor_of(a[1], "gate"), *state = tensor_of(a[4], "state");
    const at::Tensor *out = tensor_of(a[7], "out"), *out_state = tensor_of(a[8], "out_state");
    require(x, "x is needed");
    const ScanArgs c(*x, gate, a[2], a[3]);
    fo_scan n = {};
    n.batch = c.batch, n.tokens = c.tokens, n.channels = c.channels;
    n.type = type_code(c.type), n.gate_type = type_code(c.gate_type), n.decay = c.decay, n.mix = c.mix;
    n.x = c.rows(x, c.type, "x", &n.x_at);
    n.gate = c.rows(gate, c.gate_type, "gate", &n.gate_at);
    n.state = c.state(state, "state");
    n.reset = c.marks(tensor_of(a[5], "reset"), &n.reset_at);
    n.lengths = c.ends(tensor_of(a[6], "lengths"), &n.lengths_type);
    at::Tensor h, last;
    if (!out) h = make(x->sizes(), c.type, c.gpu);
    if (!out_state) last = make(c.state_sizes, c.wide, c.gpu);
    n.h = c.rows(out ? out : &h, c.type, "out", &n.h_at, out != nullptr);
    n.last = c.state(out_state ? out_state : &last, "out_state", out_state != nullptr);
    const OnGpu on(c.gpu);
    const cudaStream_t st = stream_of(c.gpu);
    const ScanScratch ws(c, st);
    check_status(fused_scan(&n, ws.at, ws.bytes, st), "fused_scan");
    if (out) written(*out);
    if (out_state) written(*out_state);
    PyObject *ho = given_or_new(a[7], h);
    return pair_of(ho, given_or_new(a[8], last));
}

// scan_grad(dh, x, gate, h, decay, mix, state, reset, lengths, dlast)
PyObject *scan_grad_impl(PyObject *const *a)
{
    const at::Tensor *dh = tensor_of(a[0], "dh"), *x = tensor_of(a[1], "x"), *gate = tensor_of(a[2], "gate"), *h = tensor_of(a[3], "h");
    const at::Tensor *state = tensor_of(a[6], "state"), *dlast = tensor_of(a[9], "dlast");
    require(h, "h is needed");
    require(dh || dlast, "dh or dlast is needed");
    const ScanArgs c(*h, gate, a[4], a[5]);
    require(x || c.mix == FO_MIX_ONE, "x is needed");
    fo_scan_grad n = {};
    n.batch = c.batch, n.tokens = c.tokens, n.channels = c.channels;
    n.type = type_code(c.type), n.gate_type = type_code(c.gate_type), n.decay = c.decay, n.mix = c.mix;
    n.dh = c.rows(dh, c.type, "dh", &n.dh_at);
    n.x = c.rows(x, c.type, "x", &n.x_at);
    n.gate = c.rows(gate, c.gate_type, "gate", &n.gate_at);
    n.h = c.rows(h, c.type, "h", &n.h_at);
    n.state = c.state(state, "state");
    n.dlast = c.state(dlast, "dlast");
    n.reset = c.marks(tensor_of(a[7], "reset"), &n.reset_at);
    n.lengths = c.ends(tensor_of(a[8], "lengths"), &n.lengths_type);
    Results got;
    const at::Tensor dx = make(h->sizes(), c.type, c.gpu), dgate = make(h->sizes(), c.gate_type, c.gpu);
    got.put("x", or_none(dx)), got.put("gate", or_none(dgate));
    n.dx = c.rows(&dx, c.type, "dx", &n.dx_at);
    n.dgate = c.rows(&dgate, c.gate_type, "dgate", &n.dgate_at);
    if (state) {
        const at::Tensor dstate = make(c.state_sizes, c.wide, c.gpu);
        got.put("state", or_none(dstate));
        n.dstate = c.state(&dstate, "dstate");
    }
    const OnGpu on(c.gpu);
    const cudaStream_t st = stream_of(c.gpu);
    const ScanScratch ws(c, st);
    check_status(fused_scan_grad(&n, ws.at, ws.bytes, st), "fused_scan_grad");
    return got.release();
}

// ------------------------------------------------------------------------------------------------------------ distillation
namespace {

struct DistillArgs {
    fo_distill n = {};
    c10::DeviceIndex gpu;
    at::ScalarType type, wide;
    int64_t rows, vocab;

    // (logits, ids, values, tail, temperature)
    explicit DistillArgs(PyObject *const *a)
    {
        const at::Tensor *z = tensor_of(a[0], "logits"), *ids = tensor_of(a[1], "ids"), *values = tensor_of(a[2], "values");
        const at::Tensor *tail = tensor_of(a[3], "tail");
        require(z && ids && values, "logits, ids and values are needed");
        gpu = gpu_of(*z);
        require(z->dim() == 2, "logits are (rows, vocab)");
        type = z->scalar_type(), wide = wide_type(type);
        rows = z->size(0), vocab = z->size(1);
        n.rows = rows, n.vocab = vocab, n.type = type_code(type), n.temperature = number(a[4]);
        n.logits = matrix(z, vocab, type, "logits", &n.ld_logits);
        require(ids->dim() == 2, "ids are (rows, entries)");
        n.top = ids->size(1), n.ids_type = int_code(*ids, "ids");
        n.ids = matrix(ids, n.top, ids->scalar_type(), "ids", &n.ld_ids);
        const at::ScalarType vt = values->scalar_type();
        require(vt == type || (vt == at::kFloat && sixteen(type)), "values have the logits' type, or float32 beside 16 bits");
        n.values_type = type_code(vt);
        n.values = matrix(values, n.top, vt, "values", &n.ld_values);
        n.tail = packed_of(tail, {rows}, wide, gpu, "tail");
    }
    void *matrix(const at::Tensor *t, int64_t cols, at::ScalarType of, const char *name, int64_t *ld, bool write = false) const
    {
        void *p = rows_of(t, {rows, cols}, of, gpu, name, write);
        *ld = rows > 1 ? t->stride(0) : cols;
        if (*ld < cols) refuse(name, ": rows overlap");
        return p;
    }
    void weights(PyObject *o) { n.dloss = packed_of(tensor_of(o, "dloss"), {rows}, wide, gpu, "dloss"); }
    at::Tensor result(PyObject *o)
    {
        const at::Tensor *given = tensor_of(o, "out");
        const at::Tensor dz = given ? *given : make({rows, vocab}, type, gpu);
        n.dz = matrix(&dz, vocab, type, "out", &n.ld_dz, given != nullptr);
        return dz;
    }
};

}  // namespace

// distill(logits, ids, values, tail, temperature, stats, step, dloss, out): step: (loss, dz), else (loss, stats or None)
PyObject *distill_impl(PyObject *const *a)
{
    DistillArgs c(a);
    const int stats = PyObject_IsTrue(a[5]), step = PyObject_IsTrue(a[6]);
    if (PyErr_Occurred()) throw Raised();
    const at::Tensor loss = make({c.rows}, c.wide, c.gpu);
    c.n.loss = c.rows ? loss.data_ptr() : nullptr;
    at::Tensor second;
    const OnGpu on(c.gpu);
    if (step) {
        c.weights(a[7]);
        second = c.result(a[8]);
        check_status(fused_distill_step(&c.n, stream_of(c.gpu)), "fused_distill_step");
        if (a[8] != Py_None) written(second);
    } else {
        if (stats) {
            second = make({3, c.rows}, c.wide, c.gpu);
            c.n.stats = c.rows ? second.data_ptr() : nullptr;
        }
        check_status(fused_distill(&c.n, stream_of(c.gpu)), "fused_distill");
    }
    PyObject *lo = or_none(loss);
    return pair_of(lo, step ? given_or_new(a[8], second) : or_none(second));
}

// distill_grad(logits, ids, values, tail, temperature, dloss, stats, out)
PyObject *distill_grad_impl(PyObject *const *a)
{
    DistillArgs c(a);
    c.weights(a[5]);
    const at::Tensor *stats = tensor_of(a[6], "stats");
    require(stats, "stats are needed");
    c.n.stats = packed_of(stats, {3, c.rows}, c.wide, c.gpu, "stats");
    const at::Tensor dz = c.result(a[7]);
    const OnGpu on(c.gpu);
    check_status(fused_distill_grad(&c.n, stream_of(c.gpu)), "fused_distill_grad");
    if (a[7] != Py_None) written(dz);
    return given_or_new(a[7], dz);
}

}  // namespace fo_py
