// Gated linear recurrence: argument checks, alignment, dispatch over element types.
#include <initializer_list>

#include "scan.cuh"

namespace fo {

#define FO_SCAN_PAIRS(X)                           \
    X(FO_F64, FO_F64, double, double)              \
    X(FO_F32, FO_F32, float, float)                \
    X(FO_BF16, FO_BF16, __nv_bfloat16, __nv_bfloat16) \
    X(FO_BF16, FO_F32, __nv_bfloat16, float)       \
    X(FO_F16, FO_F16, __half, __half)              \
    X(FO_F16, FO_F32, __half, float)

#define FO_EXTERN(t, g, T, G) extern template cudaError_t launch_scan<T, G>(ScanParams, bool, void *, cudaStream_t);
FO_SCAN_PAIRS(FO_EXTERN)
#undef FO_EXTERN

namespace {

int state_code(int type) { return type == FO_F64 ? FO_F64 : FO_F32; }

int check_scan(long long batch, long long tokens, long long channels, int type, int gate_type, int decay, int mix, const void *lengths,
               int lengths_type, std::initializer_list<fo_rows> strides)
{
    if (batch < 0 || tokens < 0 || channels < 0) return FO_ERR_SHAPE;
    if (channels > FO_SCAN_MAX_CHANNELS || tokens > FO_SCAN_MAX_TOKENS) return FO_ERR_UNSUPPORTED;
    bool ok = false;
#define FO_CASE(t, g, T, G) ok = ok || (type == t && gate_type == g);
    FO_SCAN_PAIRS(FO_CASE)
#undef FO_CASE
    if (!ok || decay < FO_DECAY_VALUE || decay > FO_DECAY_EXP || mix < FO_MIX_ONE || mix > FO_MIX_ROOT) return FO_ERR_UNSUPPORTED;
    if (lengths && lengths_type != FO_I32 && lengths_type != FO_I64) return FO_ERR_UNSUPPORTED;
    if (lengths && ((uintptr_t)lengths & (lengths_type == FO_I64 ? 7u : 3u))) return FO_ERR_UNSUPPORTED;
    for (const fo_rows &s : strides)
        if (s.batch < 0 || s.token < 0) return FO_ERR_SHAPE;
    // CTAs are counted in 31 bits
    const long long tiles = (channels + 31) / 32;
    if (tiles && batch > 0x7fffffffLL / tiles) return FO_ERR_UNSUPPORTED;
    return FO_OK;
}
bool all_on(int type, std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (!on_elements(p, type)) return false;
    return true;
}
// Every row begins at a multiple of `bytes`.
bool rows_at(const void *p, const fo_rows &s, int type, int bytes)
{
    return (((uintptr_t)p | (unsigned long long)(s.batch | s.token) * (unsigned)elem_bytes(type)) & (unsigned)(bytes - 1)) == 0;
}
int whole_if(const void *p, const fo_rows &s, int type, ScanTensor bit) { return rows_at(p, s, type, 16) ? bit : 0; }
// 16 rows of every tensor lie within 2^30 bytes, and so do their channels.
int near_if(std::initializer_list<fo_rows> strides, long long channels)
{
    for (const fo_rows &s : strides)
        if (s.token > (1LL << 30) / (16 * 8)) return 0;
    return channels <= (1LL << 27) ? kScanNear : 0;
}
int pairs_if(const void *p, const fo_rows &s, int type, ScanTensor bit) { return rows_at(p, s, type, 2 * elem_bytes(type)) ? bit : 0; }

int launch(const ScanParams &p, int type, int gate_type, bool grad, void *ws, size_t ws_bytes, cudaStream_t st)
{
    const size_t needed = fused_scan_workspace_bytes(p.tokens);
    if (needed) {
        const int rc = check_workspace(ws, ws_bytes, needed);
        if (rc != FO_OK) return rc;
    }
    cudaError_t e = cudaErrorInvalidValue;
#define FO_CASE(t, g, T, G) \
    if (type == t && gate_type == g) e = launch_scan<T, G>(p, grad, ws, st);
    FO_SCAN_PAIRS(FO_CASE)
#undef FO_CASE
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

size_t fused_scan_workspace_bytes(int64_t tokens)
{
    if (tokens < kScanLeastChunked) return 0;
    // three states and a mark of every chunk: of at most 64 channels each, and of as many as there are CTAs on all SMs
    return sizeof(WsHead) + (size_t)2 * kScanMostSms * (64 * 3 * sizeof(double) + sizeof(int));
}

int fused_scan(const fo_scan *a, void *ws, size_t ws_bytes, void *stream)
{
    if (!a) return FO_ERR_NULL;
    const int rc = check_scan(a->batch, a->tokens, a->channels, a->type, a->gate_type, a->decay, a->mix, a->lengths, a->lengths_type,
                              {a->x_at, a->gate_at, a->h_at, a->reset_at});
    if (rc != FO_OK) return rc;
    if (a->batch == 0 || a->channels == 0) return FO_OK;
    if (a->tokens > 0 && (!a->x || !a->gate || !a->h)) return FO_ERR_NULL;
    if (!all_on(a->type, {a->x, a->h}) || !all_on(a->gate_type, {a->gate}) || !all_on(state_code(a->type), {a->state, a->last}))
        return FO_ERR_UNSUPPORTED;
    if (a->tokens == 0 && !a->last) return FO_OK;
    ScanParams p = {};
    p.tokens = (int)a->tokens, p.channels = a->channels, p.batch = a->batch, p.mode = a->decay * 3 + a->mix;
    p.x = a->x, p.gate = a->gate, p.state = a->state, p.lengths = a->lengths, p.long_lengths = a->lengths_type == FO_I64;
    p.reset = static_cast<const unsigned char *>(a->reset);
    p.h = a->h, p.last = a->last;
    p.x_at = a->x_at, p.gate_at = a->gate_at, p.reset_at = a->reset_at, p.h_at = a->h_at;
    p.whole = whole_if(a->x, a->x_at, a->type, kScanX) | whole_if(a->gate, a->gate_at, a->gate_type, kScanGate)
              | pairs_if(a->h, a->h_at, a->type, kScanOut) | near_if({a->x_at, a->gate_at, a->h_at}, a->channels);
    return launch(p, a->type, a->gate_type, false, ws, ws_bytes, (cudaStream_t)stream);
}

int fused_scan_grad(const fo_scan_grad *a, void *ws, size_t ws_bytes, void *stream)
{
    if (!a) return FO_ERR_NULL;
    const int rc = check_scan(a->batch, a->tokens, a->channels, a->type, a->gate_type, a->decay, a->mix, a->lengths, a->lengths_type,
                              {a->dh_at, a->x_at, a->gate_at, a->h_at, a->reset_at, a->dx_at, a->dgate_at});
    if (rc != FO_OK) return rc;
    if (a->batch == 0 || a->channels == 0) return FO_OK;
    const bool mixes = a->mix != FO_MIX_ONE;
    if (a->tokens > 0 && ((mixes && !a->x) || !a->gate || !a->h || !a->dx || !a->dgate)) return FO_ERR_NULL;
    if (!all_on(a->type, {a->dh, a->h, a->dx}) || (mixes && !all_on(a->type, {a->x})) || !all_on(a->gate_type, {a->gate, a->dgate})
        || !all_on(state_code(a->type), {a->dlast, a->state, a->dstate}))
        return FO_ERR_UNSUPPORTED;
    if (a->tokens == 0 && !a->dstate) return FO_OK;
    ScanParams p = {};
    p.tokens = (int)a->tokens, p.channels = a->channels, p.batch = a->batch, p.mode = a->decay * 3 + a->mix;
    p.x = a->x, p.gate = a->gate, p.state = a->state, p.lengths = a->lengths, p.long_lengths = a->lengths_type == FO_I64;
    p.reset = static_cast<const unsigned char *>(a->reset);
    p.h = a->dx, p.last = a->dstate, p.dh = a->dh, p.dlast = a->dlast, p.h_in = a->h, p.dgate = a->dgate;
    p.x_at = a->x_at, p.gate_at = a->gate_at, p.reset_at = a->reset_at, p.h_at = a->dx_at;
    p.dh_at = a->dh_at, p.h_in_at = a->h_at, p.dgate_at = a->dgate_at;
    p.whole = whole_if(a->x, a->x_at, a->type, kScanX) | whole_if(a->gate, a->gate_at, a->gate_type, kScanGate)
              | whole_if(a->dh, a->dh_at, a->type, kScanDh) | whole_if(a->h, a->h_at, a->type, kScanH)
              | pairs_if(a->dx, a->dx_at, a->type, kScanOut) | pairs_if(a->dgate, a->dgate_at, a->gate_type, kScanOutGate)
              | near_if({a->x_at, a->gate_at, a->dh_at, a->h_at, a->dx_at, a->dgate_at}, a->channels);
    if (!mixes) p.whole |= kScanX;                           // not looked at
    if (!a->dh) p.whole |= kScanDh;
    return launch(p, a->type, a->gate_type, true, ws, ws_bytes, (cudaStream_t)stream);
}

}  // extern "C"
