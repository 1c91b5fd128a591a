// Distillation loss and gradient: argument checks, dispatch over element types.
#include "distill.cuh"

namespace fo {

extern template cudaError_t launch_distill<double>(DistillParams, DistillWay, cudaStream_t);
extern template cudaError_t launch_distill<float>(DistillParams, DistillWay, cudaStream_t);
extern template cudaError_t launch_distill<__nv_bfloat16>(DistillParams, DistillWay, cudaStream_t);
extern template cudaError_t launch_distill<__half>(DistillParams, DistillWay, cudaStream_t);

namespace {

int run_distill(const fo_distill *a, DistillWay way, void *stream)
{
    if (!a) return FO_ERR_NULL;
    if (a->rows < 0 || a->vocab < 0 || a->top < 0) return FO_ERR_SHAPE;
    if (a->type < FO_F64 || a->type > FO_F16 || (a->ids_type != FO_I32 && a->ids_type != FO_I64)) return FO_ERR_UNSUPPORTED;
    if (a->values_type != a->type && !(a->values_type == FO_F32 && elem_bytes(a->type) == 2)) return FO_ERR_UNSUPPORTED;
    if (!(a->temperature >= 1e-300) || a->temperature > 1e300) return FO_ERR_UNSUPPORTED;      // 1 / temperature is finite
    if (a->top > FO_DISTILL_MAX_TOP || a->rows > 0x7fffffffLL || a->vocab > FO_DISTILL_MAX_VOCAB) return FO_ERR_UNSUPPORTED;
    if (a->rows == 0) return FO_OK;
    const bool grad = way != kDistillLoss;
    if (a->ld_logits < a->vocab || a->ld_ids < a->top || a->ld_values < a->top || (grad && a->ld_dz < a->vocab)) return FO_ERR_SHAPE;
    if (a->vocab > 0 && (!a->logits || (grad && !a->dz))) return FO_ERR_NULL;
    if (a->top > 0 && (!a->ids || !a->values)) return FO_ERR_NULL;
    if ((way == kDistillStep && !a->loss) || (way == kDistillGrad && !a->stats)) return FO_ERR_NULL;
    if (way == kDistillLoss && !a->loss && !a->stats) return FO_ERR_NULL;
    const int wide = a->type == FO_F64 ? FO_F64 : FO_F32;
    if (!on_elements(a->logits, a->type) || (grad && !on_elements(a->dz, a->type)) || !on_elements(a->values, a->values_type)
        || ((uintptr_t)a->ids & (a->ids_type == FO_I64 ? 7u : 3u)) != 0 || !on_elements(a->tail, wide) || !on_elements(a->loss, wide)
        || !on_elements(a->stats, wide) || (grad && !on_elements(a->dloss, wide)))
        return FO_ERR_UNSUPPORTED;
    if (way == kDistillGrad && a->vocab == 0) return FO_OK;
    DistillParams p = {};
    p.rows = a->rows, p.vocab = (int)a->vocab, p.top = (int)a->top;
    p.ids_long = a->ids_type == FO_I64, p.wide_values = a->values_type != a->type;
    p.ld_logits = a->ld_logits, p.ld_ids = a->ld_ids, p.ld_values = a->ld_values, p.ld_dz = a->ld_dz;
    p.logits = a->logits, p.ids = a->ids, p.values = a->values, p.tail = a->tail;
    p.dloss = grad ? a->dloss : nullptr;
    p.loss = a->loss, p.stats = a->stats, p.dz = a->dz;
    p.inv_t = 1.0 / a->temperature;
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    switch (a->type) {
    case FO_F64: e = launch_distill<double>(p, way, st); break;
    case FO_F32: e = launch_distill<float>(p, way, st); break;
    case FO_BF16: e = launch_distill<__nv_bfloat16>(p, way, st); break;
    default: e = launch_distill<__half>(p, way, st); break;
    }
    return e == cudaSuccess ? FO_OK : cuda_fail(e);
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int fused_distill(const fo_distill *a, void *stream) { return run_distill(a, kDistillLoss, stream); }
int fused_distill_grad(const fo_distill *a, void *stream) { return run_distill(a, kDistillGrad, stream); }
int fused_distill_step(const fo_distill *a, void *stream) { return run_distill(a, kDistillStep, stream); }

}  // extern "C"
