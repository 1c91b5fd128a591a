// Block norm and its gradient: argument checks, alignment, dispatch over element types, and the sum
// of the gradient's column partials.
#include <initializer_list>

#include "block_norm_launch.cuh"

namespace fo {

#define FO_PAIRS(X)                                                    \
    X(FO_F64, FO_F64, double, double)                                  \
    X(FO_F32, FO_F32, float, float)                                    \
    X(FO_BF16, FO_BF16, __nv_bfloat16, __nv_bfloat16)                  \
    X(FO_F16, FO_F16, __half, __half)                                  \
    X(FO_F32, FO_BF16, float, __nv_bfloat16)                           \
    X(FO_F32, FO_F16, float, __half)

#define FO_EXTERN(s, b, TS, TB)                                                                    \
    extern template cudaError_t launch_block_norm<TS, TB>(const BlockNormParams &, cudaStream_t);  \
    extern template cudaError_t launch_block_norm_grad<TS, TB>(BlockNormGradParams, int, int *, cudaStream_t);
FO_PAIRS(FO_EXTERN)
#undef FO_EXTERN

namespace {

bool types_ok(int stream, int block, int vec)
{
    bool ok = false;
#define FO_CASE(s, b, TS, TB) ok = ok || (stream == s && block == b);
    FO_PAIRS(FO_CASE)
#undef FO_CASE
    return ok && (vec == block || (vec == FO_F32 && elem_bytes(block) == 2));
}

bool spec_ok(const fo_norm &n)
{
    return n.kind >= FO_NORM_NONE && n.kind <= FO_NORM_LAYER && (n.kind == FO_NORM_NONE || n.eps >= 0.0);
}

// Every pointer of `ps` is one to elements of a type.
bool all_on(int type, std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (!on_elements(p, type)) return false;
    return true;
}
int sum_code(int block_type) { return block_type == FO_F64 ? FO_F64 : FO_F32; }

NormSpec spec_of(const fo_norm &n)
{
    NormSpec s = {n.kind, 0, n.eps, nullptr, nullptr};
    if (n.kind != FO_NORM_NONE) s.weight = n.weight, s.bias = n.bias;
    return s;
}

// Collects whether every row of every matrix can move in pieces (16 bytes of the block's type, the same number
// of elements of the stream's), and every vector in 16 bytes.
struct Pieces {
    bool ok;
    int block_bytes;
    bool vectors = true;
    void matrix(const void *p, long long ld, int type)
    {
        const int piece = 16 * elem_bytes(type) / block_bytes;
        if (p) ok = ok && ((uintptr_t)p & (unsigned)(piece - 1)) == 0 && (ld * elem_bytes(type)) % piece == 0;
    }
    void vector(const void *p) { vectors = vectors && ((uintptr_t)p & 15u) == 0; }
    void norm(const fo_norm &n)
    {
        if (n.kind != FO_NORM_NONE) vector(n.weight), vector(n.bias);
    }
};

int check_shape(long long rows, long long cols)
{
    if (rows < 0 || cols < 0) return FO_ERR_SHAPE;
    if (cols > FO_BLOCK_NORM_MAX_COLS || rows > 0x7fffffffLL) return FO_ERR_UNSUPPORTED;
    return FO_OK;
}

// Gate and leading dimensions of the block's part.
int check_gate(const void *gate, int access, int act, long long ld, long long rows, long long cols)
{
    if (!gate) return FO_OK;
    if (access < FO_AT_CELL || access > FO_AT_COL || act < FO_ACT_LINEAR || act > FO_ACT_TANH) return FO_ERR_UNSUPPORTED;
    if (access == FO_AT_CELL && ld < cols) return FO_ERR_SHAPE;
    if (access == FO_AT_ROW && rows > 1 && ld < 1) return FO_ERR_SHAPE;
    return FO_OK;
}

// Upper bound on the CTAs (clusters) that leave a line of partial column sums: what is resident of CTAs of 256
// threads for short rows, of 512 for longer ones.
int grad_lines(long long rows, long long cols)
{
    const long long cap = cols <= 256 ? 148 * 4 : cols <= 8192 ? 148 * 2 : 148;
    const long long n = rows < cap ? rows : cap;
    return (int)(n > 1 ? n : 1);
}

// Statistics or sums over no elements are zero.
int clear_sums(void *p, long long values, int block_type, cudaStream_t st)
{
    if (!p || values == 0) return FO_OK;
    const cudaError_t e = cudaMemsetAsync(p, 0, (size_t)values * (block_type == FO_F64 ? 8 : 4), st);
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

size_t grad_line_bytes(long long rows, long long cols, int block_type)
{
    return (size_t)kGradSlots * grad_lines(rows, cols) * (size_t)cols * (block_type == FO_F64 ? 8 : 4);
}
}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int fused_block_norm(const fo_block_norm *a, void *stream)
{
    if (!a) return FO_ERR_NULL;
    int rc = check_shape(a->rows, a->cols);
    if (rc != FO_OK) return rc;
    if (!types_ok(a->stream_type, a->block_type, a->vec_type) || !spec_ok(a->post) || !spec_ok(a->pre))
        return FO_ERR_UNSUPPORTED;
    if (a->rows == 0) return FO_OK;
    if (a->cols == 0) return clear_sums(a->stats, 4 * a->rows, a->block_type, (cudaStream_t)stream);
    if (!a->x && !a->f) return FO_ERR_NULL;
    if (!a->h && !a->y && !a->stats) return FO_ERR_NULL;
    if (a->y && a->pre.kind == FO_NORM_NONE) return FO_ERR_NULL;      // y without a norm: h is that
    if (!a->f && (a->gate || a->col_scale || a->post.kind != FO_NORM_NONE)) return FO_ERR_NULL;
    if ((a->x && a->ld_x < a->cols) || (a->f && a->ld_f < a->cols) || (a->h && a->ld_h < a->cols)
        || (a->y && a->ld_y < a->cols))
        return FO_ERR_SHAPE;
    rc = check_gate(a->gate, a->gate_access, a->gate_act, a->ld_gate, a->rows, a->cols);
    if (rc != FO_OK) return rc;
    if (!all_on(a->stream_type, {a->x, a->h}) || !all_on(a->block_type, {a->f, a->gate, a->y})
        || !all_on(a->vec_type, {a->col_scale, a->post.weight, a->post.bias, a->pre.weight, a->pre.bias})
        || !all_on(sum_code(a->block_type), {a->stats}))
        return FO_ERR_UNSUPPORTED;

    BlockNormParams p = {};
    p.rows = a->rows, p.cols = (int)a->cols, p.inv_cols = 1.0 / (double)a->cols;
    p.wide_vec = a->vec_type != a->block_type;
    p.gate_access = a->gate ? a->gate_access : -1, p.gate_act = a->gate_act;
    p.x = a->x, p.f = a->f, p.gate = a->gate, p.col_scale = a->col_scale;
    p.ld_x = a->ld_x, p.ld_f = a->ld_f, p.ld_gate = a->ld_gate, p.ld_h = a->ld_h, p.ld_y = a->ld_y;
    p.scale = a->scale;
    p.post = spec_of(a->post), p.pre = spec_of(a->pre);
    p.h = a->h, p.y = a->y, p.stats = a->stats;
    Pieces all = {a->cols % (16 / elem_bytes(a->block_type)) == 0, elem_bytes(a->block_type)};
    all.matrix(a->x, a->ld_x, a->stream_type);
    all.matrix(a->h, a->ld_h, a->stream_type);
    all.matrix(a->f, a->ld_f, a->block_type);
    all.matrix(a->y, a->ld_y, a->block_type);
    if (p.gate_access == FO_AT_CELL) all.matrix(a->gate, a->ld_gate, a->block_type);
    if (p.gate_access == FO_AT_COL) all.vector(a->gate);
    all.vector(a->col_scale), all.norm(a->post), all.norm(a->pre);
    p.aligned = all.ok && all.vectors, p.vectors = all.vectors;

    cudaError_t e = cudaErrorInvalidValue;
#define FO_CASE(s, b, TS, TB) \
    if (a->stream_type == s && a->block_type == b) e = launch_block_norm<TS, TB>(p, (cudaStream_t)stream);
    FO_PAIRS(FO_CASE)
#undef FO_CASE
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

size_t fused_block_norm_grad_workspace_bytes(int64_t rows, int64_t cols, int block_type)
{
    if (check_shape(rows, cols) != FO_OK || block_type < FO_F64 || block_type > FO_F16) return 0;
    return sizeof(WsHead) + grad_line_bytes(rows, cols, block_type);
}

int fused_block_norm_grad(const fo_block_norm_grad *a, void *ws, size_t ws_bytes, void *stream)
{
    if (!a) return FO_ERR_NULL;
    int rc = check_shape(a->rows, a->cols);
    if (rc != FO_OK) return rc;
    if (!types_ok(a->stream_type, a->block_type, a->vec_type) || !spec_ok(a->post) || !spec_ok(a->pre))
        return FO_ERR_UNSUPPORTED;
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->cols == 0) return clear_sums(a->gate_access == FO_AT_ROW ? a->dgate : nullptr, a->rows, a->block_type, st);
    void *const sums[kGradSlots] = {a->dpre_weight, a->dpre_bias, a->dpost_weight, a->dpost_bias, a->dcol_scale,
                                    a->gate_access == FO_AT_COL ? a->dgate : nullptr};
    if (a->rows == 0) {                                        // sums over no rows; nothing else has a size
        for (void *s : sums)
            if ((rc = clear_sums(s, a->cols, a->block_type, st)) != FO_OK) return rc;
        return FO_OK;
    }
    const bool pre = a->dy != nullptr, post = a->f && a->post.kind != FO_NORM_NONE;
    if (!a->dh && !a->dy) return FO_ERR_NULL;
    if (pre && (a->pre.kind == FO_NORM_NONE || !a->h)) return FO_ERR_NULL;
    if ((pre || post) && !a->stats) return FO_ERR_NULL;
    if (!a->f && (a->gate || a->col_scale || a->post.kind != FO_NORM_NONE || a->df || a->dgate || a->dcol_scale
                  || a->dpost_weight || a->dpost_bias))
        return FO_ERR_NULL;
    if ((a->dgate && !a->gate) || (!post && (a->dpost_weight || a->dpost_bias))
        || (a->pre.kind == FO_NORM_NONE && (a->dpre_weight || a->dpre_bias)))
        return FO_ERR_NULL;
    if ((a->dh && a->ld_dh < a->cols) || (pre && (a->ld_dy < a->cols || a->ld_h < a->cols)) || (a->f && a->ld_f < a->cols)
        || (a->dx && a->ld_dx < a->cols) || (a->df && a->ld_df < a->cols)
        || (a->dgate && a->gate_access == FO_AT_CELL && a->ld_dgate < a->cols))
        return FO_ERR_SHAPE;
    rc = check_gate(a->gate, a->gate_access, a->gate_act, a->ld_gate, a->rows, a->cols);
    if (rc != FO_OK) return rc;
    const int dgate_type = a->gate_access == FO_AT_CELL ? a->block_type : sum_code(a->block_type);
    if (!all_on(a->stream_type, {a->dh, a->h, a->dx}) || !all_on(a->block_type, {a->dy, a->f, a->gate, a->df})
        || !all_on(a->vec_type, {a->col_scale, a->post.weight, a->post.bias, a->pre.weight, a->pre.bias})
        || !all_on(sum_code(a->block_type), {a->stats, a->dcol_scale, a->dpost_weight, a->dpost_bias, a->dpre_weight, a->dpre_bias})
        || !all_on(dgate_type, {a->dgate}))
        return FO_ERR_UNSUPPORTED;
    rc = check_workspace(ws, ws_bytes, fused_block_norm_grad_workspace_bytes(a->rows, a->cols, a->block_type));
    if (rc != FO_OK) return rc;
    BlockNormGradParams p = {};
    p.rows = a->rows, p.cols = (int)a->cols, p.inv_cols = 1.0 / (double)a->cols;
    p.wide_vec = a->vec_type != a->block_type;
    p.gate_access = a->gate ? a->gate_access : -1, p.gate_act = a->gate_act;
    p.dh = a->dh, p.dy = a->dy, p.h = a->h, p.f = a->f, p.gate = a->gate, p.col_scale = a->col_scale, p.stats = a->stats;
    p.ld_dh = a->ld_dh, p.ld_dy = a->ld_dy, p.ld_h = a->ld_h, p.ld_f = a->ld_f, p.ld_gate = a->ld_gate;
    p.scale = a->scale;
    p.post = spec_of(a->post), p.pre = spec_of(a->pre);
    p.dx = a->dx, p.df = a->df, p.dgate = p.gate_access == FO_AT_COL ? nullptr : a->dgate;
    p.ld_dx = a->ld_dx, p.ld_df = a->ld_df, p.ld_dgate = a->ld_dgate;
    p.partial = static_cast<char *>(ws) + sizeof(WsHead);
    Pieces all = {a->cols % (16 / elem_bytes(a->block_type)) == 0, elem_bytes(a->block_type)};
    all.matrix(a->dh, a->ld_dh, a->stream_type);
    all.matrix(a->dx, a->ld_dx, a->stream_type);
    if (pre) all.matrix(a->h, a->ld_h, a->stream_type), all.matrix(a->dy, a->ld_dy, a->block_type);
    all.matrix(a->f, a->ld_f, a->block_type);
    all.matrix(a->df, a->ld_df, a->block_type);
    if (p.gate_access == FO_AT_CELL) all.matrix(a->gate, a->ld_gate, a->block_type);
    if (p.gate_access == FO_AT_CELL) all.matrix(a->dgate, a->ld_dgate, a->block_type);
    if (p.gate_access == FO_AT_COL) all.vector(a->gate);
    all.vector(a->col_scale), all.norm(a->post), all.norm(a->pre);
    p.aligned = all.ok && all.vectors, p.vectors = all.vectors;

    int n_sums = 0;
    ColumnSumParams cs = {};
    for (int s = 0; s < kGradSlots; ++s) {
        if (!sums[s]) continue;
        p.slots |= 1u << s;
        cs.out[n_sums++] = sums[s];
    }
    int lines = 0;
    cudaError_t e = cudaErrorInvalidValue;
#define FO_CASE(s, b, TS, TB) \
    if (a->stream_type == s && a->block_type == b) e = launch_block_norm_grad<TS, TB>(p, grad_lines(a->rows, a->cols), &lines, st);
    FO_PAIRS(FO_CASE)
#undef FO_CASE
    if (e == cudaSuccess && n_sums > 0) {
        cs.partial = p.partial, cs.lines = lines, cs.cols = p.cols;
        const dim3 grid((unsigned)((a->cols + 31) / 32), (unsigned)n_sums);
        e = a->block_type == FO_F64 ? launch_beside(column_sum_kernel<double>, grid, kSumWarps * 32, st, cs)
                                    : launch_beside(column_sum_kernel<float>, grid, kSumWarps * 32, st, cs);
    }
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

}  // extern "C"
