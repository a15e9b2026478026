// C ABI entry points of the training-side calls: argument validation and path selection.
#include <math.h>

#include "sr_train.cuh"

using namespace sr;

namespace {

bool on(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

cudaError_t run_grad(const GradArgs& a)
{
    const bool sums = a.gdict || a.ggamma;
    if (grad_roles_supported(a)) {
        int slots = 0;
        if (cudaError_t e = launch_grad_roles(a, &slots)) return e;
        return sums ? launch_grad_dict_sum(a, slots) : cudaSuccess;
    }
    if (a.gcoef)
        if (cudaError_t e = grad_coef_tc_supported(a) ? launch_grad_coef_tc(a) : launch_grad_coef_fma(a)) return e;
    if (sums) {
        int slots = 0;
        if (cudaError_t e = grad_dict_tc_supported(a) ? launch_grad_dict_tc(a, &slots) : launch_grad_dict_fma(a, &slots)) return e;
        return launch_grad_dict_sum(a, slots);
    }
    return cudaSuccess;
}

size_t grad_scratch_bytes(const sr_dims* d) { return (size_t)grad_slots() * d->D * d->k * d->k * sizeof(float); }

int grad_call(int mode, const float* lr, const void* coef, int coef_dtype, const uint8_t* idx, const float* gamma, const float* dict,
              const float* gout, void* gcoef, float* gdict, float* ggamma, const sr_dims* d, int s, uint32_t flags, void* scratch,
              size_t scratch_bytes, void* stream)
{
    const size_t esz = coef_dtype == SR_F16 ? 2 : 4;
    const bool sums = gdict || ggamma;
    if (sums && (!coef || !scratch)) return SR_ERR_NULL;
    if (!on(lr, 4) || !on(dict, 4) || !on(gout, 4) || !on(gamma, 4) || !on(coef, esz) || !on(gcoef, esz) || !on(gdict, 4) || !on(ggamma, 4) ||
        (sums && !on(scratch, 16)))
        return SR_ERR_ALIGN;
    if (sums && scratch_bytes < grad_scratch_bytes(d)) return SR_ERR_SHAPE;
    const GradArgs a{mode, lr, coef, coef_dtype, idx, gamma, dict, gout, gcoef, gdict, ggamma, static_cast<float*>(scratch),
                     make_problem(d, s, flags), (cudaStream_t)stream};
    return run_grad(a) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

int check_select(const sr_dims* d, int coef_dtype, sr_dims& dd)
{
    dd = *d;
    dd.c = 1; dd.k = 1;
    if (int e = check_dims(&dd, true)) return e;
    return coef_dtype != SR_F32 && coef_dtype != SR_F16 ? SR_ERR_UNSUPPORTED : SR_OK;
}

} // namespace

extern "C" {

size_t sr_dict_regress_grad_scratch_bytes(const sr_dims* d)
{
    return check_dims(d, true) == SR_OK ? grad_scratch_bytes(d) : 0;
}

int sr_dict_regress_dense_grad(const float* lr, const void* coef, int coef_dtype, const float* dict, const float* grad_out,
                               void* grad_coef, float* grad_dict, const sr_dims* d, uint32_t flags, void* scratch,
                               size_t scratch_bytes, void* stream)
{
    if (!lr || !dict || !grad_out || !d || (!grad_coef && !grad_dict)) return SR_ERR_NULL;
    if (int e = check_dims(d, true)) return e;
    if (coef_dtype != SR_F32 && coef_dtype != SR_F16) return SR_ERR_UNSUPPORTED;
    if (flags & ~(uint32_t)SR_UPSAMPLE_BILINEAR) return SR_ERR_UNSUPPORTED;
    return grad_call(kModeDense, lr, coef, coef_dtype, nullptr, nullptr, dict, grad_out, grad_coef, grad_dict, nullptr, d, d->D, flags, scratch,
                     scratch_bytes, stream);
}

int sr_dict_regress_selected_grad(const float* lr, const void* coef_or_sel, int coef_dtype, const uint8_t* idx, const float* gamma,
                                  const float* dict, const float* grad_out, void* grad_coef_or_sel, float* grad_dict,
                                  float* grad_gamma, const sr_dims* d, int s, uint32_t flags, void* scratch, size_t scratch_bytes,
                                  void* stream)
{
    if (!lr || !idx || !dict || !grad_out || !d || (!grad_coef_or_sel && !grad_dict && !grad_gamma)) return SR_ERR_NULL;
    if (int e = check_dims(d, true)) return e;
    if (coef_dtype != SR_F32 && coef_dtype != SR_F16) return SR_ERR_UNSUPPORTED;
    if (flags & ~(uint32_t)(SR_UPSAMPLE_BILINEAR | SR_IDX_GLOBAL | SR_COEF_COMPACT)) return SR_ERR_UNSUPPORTED;
    if (s < 1 || s > d->D) return SR_ERR_SHAPE;
    if ((gamma || grad_gamma) && !(flags & SR_IDX_GLOBAL)) return SR_ERR_UNSUPPORTED;
    const int mode = (flags & SR_IDX_GLOBAL) ? kModeGlobal : ((flags & SR_COEF_COMPACT) ? kModeCompact : kModeIdx);
    return grad_call(mode, lr, coef_or_sel, coef_dtype, idx, gamma, dict, grad_out, grad_coef_or_sel, grad_dict, grad_gamma, d, s, flags,
                     scratch, scratch_bytes, stream);
}

size_t sr_select_balance_scratch_bytes(const sr_dims* d)
{
    sr_dims dd;
    if (!d || check_select(d, SR_F32, dd) != SR_OK) return 0;
    return balance_scratch_bytes(d->n, d->D, (int64_t)d->h * d->scale * d->w * d->scale);
}

int sr_select_balance(const void* coef, int coef_dtype, const uint8_t* idx, const uint8_t* mask, float* loss, int32_t* counts,
                      float* share, float* slope, const sr_dims* d, int s, uint32_t flags, void* scratch, size_t scratch_bytes,
                      void* stream)
{
    if (!coef || !idx || !loss || !counts || !share || !slope || !d || !scratch) return SR_ERR_NULL;
    sr_dims dd;
    if (int e = check_select(d, coef_dtype, dd)) return e;
    if (flags & ~(uint32_t)SR_BALANCE_PER_FRAME) return SR_ERR_UNSUPPORTED;
    if (s < 1 || s > d->D) return SR_ERR_SHAPE;
    if (!on(coef, coef_dtype == SR_F16 ? 2 : 4) || !on(loss, 4) || !on(counts, 4) || !on(share, 4) || !on(slope, 4) || !on(scratch, 16))
        return SR_ERR_ALIGN;
    if (scratch_bytes < sr_select_balance_scratch_bytes(d)) return SR_ERR_SHAPE;
    const BalanceArgs a{coef, coef_dtype, idx, mask, loss, counts, share, slope, scratch, d->n, d->D, s,
                        (int64_t)d->h * d->scale * d->w * d->scale, (flags & SR_BALANCE_PER_FRAME) != 0, (cudaStream_t)stream};
    return launch_balance(a) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

int sr_select_balance_grad(const void* coef, int coef_dtype, const uint8_t* mask, const float* slope, const float* grad_loss,
                           float weight, void* grad_coef, const sr_dims* d, uint32_t flags, void* stream)
{
    if (!coef || !slope || !grad_coef || !d) return SR_ERR_NULL;
    sr_dims dd;
    if (int e = check_select(d, coef_dtype, dd)) return e;
    if (flags & ~(uint32_t)SR_GRAD_ADD) return SR_ERR_UNSUPPORTED;
    const size_t esz = coef_dtype == SR_F16 ? 2 : 4;
    if (!on(coef, esz) || !on(grad_coef, esz) || !on(slope, 4) || !on(grad_loss, 4)) return SR_ERR_ALIGN;
    BalanceArgs a{};
    a.coef = coef; a.coef_dtype = coef_dtype; a.mask = mask; a.n = d->n; a.D = d->D;
    a.HW = (int64_t)d->h * d->scale * d->w * d->scale;
    a.st = (cudaStream_t)stream;
    return launch_balance_grad(a, slope, grad_loss, weight, grad_coef, (flags & SR_GRAD_ADD) != 0) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

int sr_adamw_step(const sr_adamw_tensor* tensors, int32_t count, int param_dtype, int grad_dtype, int state_bits,
                  const sr_adamw_opts* o, void* stream)
{
    if (!o || (!tensors && count > 0)) return SR_ERR_NULL;
    if (count < 0) return SR_ERR_SHAPE;
    if (param_dtype < SR_F32 || param_dtype > SR_BF16 || grad_dtype < SR_F32 || grad_dtype > SR_BF16) return SR_ERR_UNSUPPORTED;
    if (state_bits != 8 && state_bits != 32) return SR_ERR_UNSUPPORTED;
    // (written so that a NaN is refused too)
    if (!(o->beta1 >= 0.0 && o->beta1 < 1.0) || !(o->beta2 >= 0.0 && o->beta2 < 1.0) || !(o->eps >= 0.0) || !isfinite(o->eps) ||
        !isfinite(o->weight_decay) || !isfinite(o->grad_scale) || (!o->lr_dev && !isfinite(o->lr)) || (!o->step_dev && o->step < 1))
        return SR_ERR_SHAPE;
    if (!on(o->lr_dev, 4) || !on(o->step_dev, 8) || !on(o->skip_dev, 4)) return SR_ERR_ALIGN;
    const size_t pe = param_dtype == SR_F32 ? 4 : 2, ge = grad_dtype == SR_F32 ? 4 : 2, se = state_bits == 8 ? 1 : 4;
    for (int32_t i = 0; i < count; ++i) {
        const sr_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n > ((int64_t)1 << 40)) return SR_ERR_SHAPE;
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v || (state_bits == 8 && (!t.m_scale || !t.v_scale))) return SR_ERR_NULL;
        if (!on(t.param, pe) || !on(t.grad, ge) || !on(t.m, se) || !on(t.v, se) || (state_bits == 8 && (!on(t.m_scale, 4) || !on(t.v_scale, 4))))
            return SR_ERR_ALIGN;
    }
    return launch_adamw(tensors, count, param_dtype, grad_dtype, state_bits, *o, (cudaStream_t)stream) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

} // extern "C"
