// Head norms with rotation: argument checks, how a call is cut into tasks, dispatch over element types, and the sum of the
// gradient's lines.
#include <algorithm>
#include <initializer_list>

#include "head_norm.cuh"

namespace fo {

extern template cudaError_t launch_head_norm<double>(const HeadParams &, int, int, bool, bool, int, cudaStream_t);
extern template cudaError_t launch_head_norm<float>(const HeadParams &, int, int, bool, bool, int, cudaStream_t);
extern template cudaError_t launch_head_norm<__nv_bfloat16>(const HeadParams &, int, int, bool, bool, int, cudaStream_t);
extern template cudaError_t launch_head_norm<__half>(const HeadParams &, int, int, bool, bool, int, cudaStream_t);

namespace {

constexpr int kSumWarps = 32;
constexpr int kHeadCtas = 2;            // CTAs per SM: as many as work at once
constexpr int kMostSms = 256;           // bound of the workspace, whatever the GPU

int wide_code(int type) { return type == FO_F64 ? FO_F64 : FO_F32; }
bool on_ints(const void *p, int type) { return ((uintptr_t)p & (type == FO_I64 ? 7u : 3u)) == 0; }

struct HeadSumParams {
    const void *partial[4];
    void *out[4];
    int lines[4];
    int dim;
};

template <class A>
__global__ void __launch_bounds__(kSumWarps * 32) head_sum_kernel(const __grid_constant__ HeadSumParams p)
{
    __shared__ A sum[kSumWarps][33];
    wait_for_earlier();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane, k = blockIdx.y;
    const A *src = static_cast<const A *>(p.partial[k]);
    A v = A(0);
    if (j < p.dim)
#pragma unroll 8
        for (int g = warp; g < p.lines[k]; g += kSumWarps) v += __ldcg(src + (size_t)g * p.dim + j);
    sum[warp][lane] = v;
    __syncthreads();
    v = sum[lane][warp];                                     // warp w: column w
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0 && blockIdx.x * 32 + warp < (unsigned)p.dim) static_cast<A *>(p.out[k])[blockIdx.x * 32 + warp] = v;
}

// The largest piece (16 bytes, 8 bytes of 16-bit types, or one element) at whose multiples every vector begins and every part of
// it that moves together lies.
struct HeadPieces {
    int bytes;
    unsigned long long all = 0;
    explicit HeadPieces(int type) : bytes(elem_bytes(type)) {}
    void tensor(const void *p, const fo_strides &s)
    {
        all |= (uintptr_t)p | (unsigned long long)(s.batch | s.token | s.head) * (unsigned)bytes;
    }
    void part(long long elements) { all |= (unsigned long long)elements * (unsigned)bytes; }
    int choose(int dim) const
    {
        if (all % 16 == 0) return 16 / bytes;
        return bytes == 2 && all % 8 == 0 && dim <= 256 ? 4 : 1;
    }
};

bool norm_ok(const fo_norm &n)
{
    return n.kind >= FO_NORM_NONE && n.kind <= FO_NORM_LAYER && (n.kind == FO_NORM_NONE || n.eps >= 0.0);
}
bool strides_ok(const fo_strides &s) { return s.batch >= 0 && s.token >= 0 && s.head >= 0; }

int check_rotation(const fo_rotation &r, int dim, int type)
{
    if (r.pairs == 0) return FO_OK;
    if (r.pairs < 0 || r.pairs > dim / 2) return FO_ERR_SHAPE;
    if ((r.pairing != FO_PAIR_HALVES && r.pairing != FO_PAIR_NEIGHBOURS) || r.axes < 1 || r.axes > FO_MAX_AXES
        || (r.position_type != FO_I32 && r.position_type != FO_I64))
        return FO_ERR_UNSUPPORTED;
    long long sum = 0;
    for (int k = 0; k < r.axes; ++k) {
        if (r.section[k] < 0) return FO_ERR_SHAPE;
        sum += r.section[k];
    }
    if (r.rows > 0x7fffffffLL) return FO_ERR_UNSUPPORTED;
    if (sum != r.pairs || r.rows < 0 || r.ld_cos < r.pairs || r.ld_sin < r.pairs || r.position_axis < 0 || r.position_batch < 0
        || r.position_token < 0)
        return FO_ERR_SHAPE;
    if (!r.positions || (r.rows > 0 && (!r.cos_table || !r.sin_table))) return FO_ERR_NULL;
    if (!on_elements(r.cos_table, wide_code(type)) || !on_elements(r.sin_table, wide_code(type))
        || !on_ints(r.positions, r.position_type))
        return FO_ERR_UNSUPPORTED;
    return FO_OK;
}

int check_sizes(long long batch, long long tokens, int dim, int type, int vec_type, int count)
{
    if (batch < 0 || tokens < 0 || dim < 0) return FO_ERR_SHAPE;
    if (dim > FO_HEAD_MAX_DIM || count < 1 || count > 2 || type < FO_F64 || type > FO_F16) return FO_ERR_UNSUPPORTED;
    if (vec_type != type && !(vec_type == FO_F32 && elem_bytes(type) == 2)) return FO_ERR_UNSUPPORTED;
    return FO_OK;
}
// heads of one tensor, and that the call's vectors can be counted in 31 bits
int check_count(long long batch, long long tokens, long long heads)
{
    if (heads < 0) return FO_ERR_SHAPE;
    const long long most = 0x7fffffffLL;
    if (batch > most || tokens > most || heads > most) return FO_ERR_UNSUPPORTED;
    if (batch && tokens && heads && (batch * tokens > most || batch * tokens * heads > most)) return FO_ERR_UNSUPPORTED;
    return FO_OK;
}

// What forward and gradient share.  `items` of a vector are spread over its lanes.
void set_rotation(HeadParams &p, const fo_rotation &r, int type, int piece)
{
    p.pairs = r.pairs;
    if (!r.pairs) return;
    // values in one load: of a piece's pairs, which are as many as its elements or half of them
    const int table = 16 / elem_bytes(wide_code(type)), width = std::max(1, std::min(table, r.pairing == FO_PAIR_HALVES ? piece : piece / 2));
    p.axes = r.axes, p.rows = r.rows, p.ld_cos = r.ld_cos, p.ld_sin = r.ld_sin;
    p.cos_table = r.cos_table, p.sin_table = r.sin_table, p.positions = r.positions;
    p.position_axis = r.position_axis, p.position_batch = r.position_batch, p.position_token = r.position_token;
    p.long_positions = r.position_type == FO_I64;
    bool whole = r.pairs % width == 0 && r.ld_cos % table == 0 && r.ld_sin % table == 0
                 && (((uintptr_t)r.cos_table | (uintptr_t)r.sin_table) & 15u) == 0;
    int end = 0;
    for (int k = 0; k < FO_MAX_AXES; ++k) {
        if (k < r.axes) end += r.section[k], whole = whole && end % width == 0;
        p.section_end[k] = end;
    }
    p.table_pieces = whole;
}

// A vector's lanes: a power of two that holds its items, 32 with as many items a lane as the kernel has.
int head_lanes(int dim, int piece)
{
    const int items = (dim + 2 * piece - 1) / (2 * piece);
    int lanes = 1;
    while (lanes < items && lanes < 32) lanes *= 2;
    return lanes;
}

// Cuts a call into turns of the warps, the same number for each, and gives the tensors CTAs by their work.  Returns the grid.
int cut(HeadParams &p, int count, long long batch, long long tokens, int sms)
{
    const long long groups = 32 / p.lanes;                   // (tokens and heads come near 2^31)
    p.tokens = (int)std::max<long long>(tokens, 1), p.all_tokens = (int)(batch * tokens);
    const long long warps = (long long)sms * kHeadCtas * kHeadWarps;
    long long wide = 0, narrow = 0, ctas[2] = {0, 0}, cost[2] = {0, 0};
    for (int k = 0; k < count; ++k)
        wide += (p.all_tokens + groups - 1) / groups * p.t[k].heads, narrow += p.all_tokens * ((p.t[k].heads + groups - 1) / groups);
    // Blocks of several tokens, whose cosines and sines serve as many turns as there are heads, where that leaves every warp four turns
    // (40 heads of 128 in bfloat16: 1024 tokens 8 us both ways, 4096 tokens 19 against 21, backwards 33 and 35), or at least one
    // and a quarter of the turns less, because heads do not come out even with the groups (7 heads of 64, 4000 tokens: 5.5 and 9.1).  With
    // few tokens the heads of one are side by side: a decoding step of 4 tokens is 40 warps of one turn, not one of 40; and so it is, however
    // many heads, where the tokens leave groups idle (200000 heads of 64 of one token 12 us, in blocks of tokens 66).
    p.wide = (wide >= 4 * warps && 4 * wide <= 5 * narrow) || (wide >= warps && 4 * wide <= 3 * narrow);
    for (int k = 0; k < count; ++k) {
        HeadTensor &t = p.t[k];
        t.blocks = p.wide ? (int)((p.all_tokens + groups - 1) / groups) : p.all_tokens;
        t.turns = p.wide ? t.heads : (int)((t.heads + groups - 1) / groups);
        // a block costs its turns and, for the cosines and sines, about one more
        cost[k] = t.turns ? t.blocks * (t.turns + 1LL) : 0;
    }
    for (int k = 0; k < count; ++k) {
        HeadTensor &t = p.t[k];
        const long long turns = (long long)t.blocks * t.turns;
        const long long share = std::max<long long>(1, (long long)sms * kHeadCtas * cost[k] / std::max<long long>(1, cost[0] + cost[1]));
        ctas[k] = std::min((turns + kHeadWarps - 1) / kHeadWarps, share);
        if (ctas[k]) t.each = (int)((turns + ctas[k] * kHeadWarps - 1) / (ctas[k] * kHeadWarps));
        else t.turns = 1;
    }
    p.ctas0 = (int)ctas[0];
    return (int)(ctas[0] + ctas[1]);
}

cudaError_t dispatch(const HeadParams &p, int type, int piece, int pairing, bool grad, bool bias, int grid, cudaStream_t st)
{
    switch (type) {
    case FO_F64: return launch_head_norm<double>(p, piece, pairing, grad, bias, grid, st);
    case FO_F32: return launch_head_norm<float>(p, piece, pairing, grad, bias, grid, st);
    case FO_BF16: return launch_head_norm<__nv_bfloat16>(p, piece, pairing, grad, bias, grid, st);
    default: return launch_head_norm<__half>(p, piece, pairing, grad, bias, grid, st);
    }
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int fused_head_norm(const fo_head_norm *a, void *stream)
{
    if (!a) return FO_ERR_NULL;
    int rc = check_sizes(a->batch, a->tokens, a->dim, a->type, a->vec_type, a->count);
    if (rc == FO_OK) rc = check_rotation(a->rotation, a->dim, a->type);
    if (rc != FO_OK) return rc;
    HeadParams p = {};
    HeadPieces pieces(a->type);
    long long vectors = 0;
    for (int k = 0; k < a->count; ++k) {
        const fo_heads &t = a->t[k];
        if ((rc = check_count(a->batch, a->tokens, t.heads)) != FO_OK) return rc;
        if (!norm_ok(t.norm)) return FO_ERR_UNSUPPORTED;
        if (!strides_ok(t.x_at) || !strides_ok(t.y_at)) return FO_ERR_SHAPE;
        if (a->batch && a->tokens && a->dim && t.heads && (!t.x || !t.y)) return FO_ERR_NULL;
        if (!on_elements(t.x, a->type) || !on_elements(t.y, a->type)
            || (t.norm.kind != FO_NORM_NONE && (!on_elements(t.norm.weight, a->vec_type) || !on_elements(t.norm.bias, a->vec_type))))
            return FO_ERR_UNSUPPORTED;
        pieces.tensor(t.x, t.x_at), pieces.tensor(t.y, t.y_at);
        HeadTensor &h = p.t[k];
        h.x = t.x, h.y = t.y, h.x_at = t.x_at, h.y_at = t.y_at, h.heads = (int)t.heads, h.kind = t.norm.kind;
        h.eps = t.norm.eps;
        if (h.kind != FO_NORM_NONE) h.weight = t.norm.weight, h.bias = t.norm.bias;
        vectors += a->batch * a->tokens * t.heads;
    }
    if (vectors == 0 || a->dim == 0) return FO_OK;
    pieces.part(a->dim), pieces.part(a->rotation.pairing == FO_PAIR_HALVES ? a->rotation.pairs : 2 * a->rotation.pairs);
    const int piece = pieces.choose(a->dim), sms = sm_count();
    if (sms <= 0) return cuda_fail(cudaErrorNoDevice);
    p.dim = a->dim, p.inv_dim = 1.0 / a->dim, p.wide_vec = a->vec_type != a->type;
    p.lanes = head_lanes(a->dim, piece);
    set_rotation(p, a->rotation, a->type, piece);
    const int grid = cut(p, a->count, a->batch, a->tokens, sms);
    const cudaError_t e = dispatch(p, a->type, piece, a->rotation.pairing, false, false, grid, (cudaStream_t)stream);
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

size_t fused_head_norm_grad_workspace_bytes(int dim, int type)
{
    if (dim < 0 || dim > FO_HEAD_MAX_DIM || type < FO_F64 || type > FO_F16) return 0;
    return sizeof(WsHead) + (size_t)(kMostSms * kHeadCtas + 2) * 2 * dim * (type == FO_F64 ? 8 : 4);
}

int fused_head_norm_grad(const fo_head_norm_grad *a, void *ws, size_t ws_bytes, void *stream)
{
    if (!a) return FO_ERR_NULL;
    int rc = check_sizes(a->batch, a->tokens, a->dim, a->type, a->vec_type, a->count);
    if (rc == FO_OK) rc = check_rotation(a->rotation, a->dim, a->type);
    if (rc != FO_OK) return rc;
    HeadParams p = {};
    HeadPieces pieces(a->type);
    const cudaStream_t st = (cudaStream_t)stream;
    long long vectors = 0;
    bool bias = false, sums = false;
    for (int k = 0; k < a->count; ++k) {
        const fo_heads_grad &t = a->t[k];
        if ((rc = check_count(a->batch, a->tokens, t.heads)) != FO_OK) return rc;
        if (!norm_ok(t.norm)) return FO_ERR_UNSUPPORTED;
        const bool normed = t.norm.kind != FO_NORM_NONE;
        if (!strides_ok(t.dy_at) || (normed && !strides_ok(t.x_at)) || !strides_ok(t.dx_at)) return FO_ERR_SHAPE;
        if (a->batch && a->tokens && a->dim && t.heads && (!t.dy || !t.dx || (normed && !t.x))) return FO_ERR_NULL;
        if (!normed && (t.dweight || t.dbias)) return FO_ERR_NULL;
        if (!on_elements(t.dy, a->type) || !on_elements(t.dx, a->type) || !on_elements(t.dweight, wide_code(a->type))
            || !on_elements(t.dbias, wide_code(a->type))
            || (normed && (!on_elements(t.x, a->type) || !on_elements(t.norm.weight, a->vec_type)
                           || !on_elements(t.norm.bias, a->vec_type))))
            return FO_ERR_UNSUPPORTED;
        pieces.tensor(t.dy, t.dy_at), pieces.tensor(t.dx, t.dx_at);
        HeadTensor &h = p.t[k];
        h.dy = t.dy, h.y = t.dx, h.dy_at = t.dy_at, h.y_at = t.dx_at, h.heads = (int)t.heads, h.kind = t.norm.kind;
        h.eps = t.norm.eps;
        if (normed) {
            pieces.tensor(t.x, t.x_at);
            h.x = t.x, h.x_at = t.x_at, h.weight = t.norm.weight;
            bias = bias || t.dbias, sums = sums || t.dweight || t.dbias;
        }
        vectors += a->batch * a->tokens * t.heads;
    }
    const int sum_bytes = a->type == FO_F64 ? 8 : 4;
    if (a->dim == 0) return FO_OK;
    // the sums of a tensor without vectors
    for (int k = 0; k < a->count; ++k)
        if (a->batch == 0 || a->tokens == 0 || a->t[k].heads == 0)
            for (void *out : {a->t[k].dweight, a->t[k].dbias})
                if (out) {
                    const cudaError_t e = cudaMemsetAsync(out, 0, (size_t)a->dim * sum_bytes, st);
                    if (e != cudaSuccess) return cuda_fail(e);
                }
    if (vectors == 0) return FO_OK;
    pieces.part(a->dim), pieces.part(a->rotation.pairing == FO_PAIR_HALVES ? a->rotation.pairs : 2 * a->rotation.pairs);
    const int piece = pieces.choose(a->dim), sms = sm_count();
    if (sms <= 0) return cuda_fail(cudaErrorNoDevice);
    p.dim = a->dim, p.inv_dim = 1.0 / a->dim, p.wide_vec = a->vec_type != a->type;
    p.lanes = head_lanes(a->dim, piece);
    set_rotation(p, a->rotation, a->type, piece);
    const int grid = cut(p, a->count, a->batch, a->tokens, std::min(sms, kMostSms));
    HeadSumParams s = {};
    int n = 0;
    if (sums) {
        rc = check_workspace(ws, ws_bytes, fused_head_norm_grad_workspace_bytes(a->dim, a->type));
        if (rc != FO_OK) return rc;
        char *at = static_cast<char *>(ws) + sizeof(WsHead);
        for (int k = 0; k < a->count; ++k) {
            const int lines = k ? grid - p.ctas0 : p.ctas0;
            auto take = [&](void *out, void **partial) {
                if (!out || lines == 0) return;
                *partial = at;
                s.partial[n] = at, s.out[n] = out, s.lines[n] = lines, ++n;
                at += (size_t)lines * a->dim * sum_bytes;
            };
            take(a->t[k].dweight, &p.t[k].partial_w);
            take(a->t[k].dbias, &p.t[k].partial_b);
        }
        s.dim = a->dim;
    }
    cudaError_t e = dispatch(p, a->type, piece, a->rotation.pairing, true, bias, grid, st);
    if (e == cudaSuccess && n > 0) {
        const dim3 sum_grid((unsigned)((a->dim + 31) / 32), (unsigned)n);
        e = a->type == FO_F64 ? launch_beside(head_sum_kernel<double>, sum_grid, kSumWarps * 32, st, s)
                              : launch_beside(head_sum_kernel<float>, sum_grid, kSumWarps * 32, st, s);
    }
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

}  // extern "C"
