// Launchers of the training-side calls: gradients of the regression, balance loss of a selection, optimiser step.
#pragma once

#include "sr_common.cuh"

namespace sr {

// Validation and problem set-up shared by the C entry points (sr_api.cu).
int check_dims(const sr_dims* d, bool need_kD);
Problem make_problem(const sr_dims* d, int s, uint32_t flags);

// One gradient call. mode: kModeDense, kModeIdx, kModeCompact or kModeGlobal; pb.s = planes of the coefficient gradient that
// are not zero (D when dense).
struct GradArgs {
    int mode;
    const float* lr;
    const void* coef;          // may be nullptr when gdict and ggamma are
    int coef_dtype;
    const uint8_t* idx;
    const float* gamma;
    const float* dict;
    const float* gout;
    void* gcoef;               // nullptr: not asked for
    float* gdict;              // nullptr: not asked for
    float* ggamma;             // nullptr: not asked for
    float* scratch;            // partial sums of gdict / ggamma, [slots][planes][k*k]
    Problem pb;
    cudaStream_t st;
};

// Partial sums of the dictionary's gradient that may be in flight: blocks of its kernels, two per multiprocessor.
inline int grad_slots() { return 2 * sm_count(); }
// Rows of one partial sum: atoms, or planes of the subset.
inline int grad_rows(const GradArgs& a) { return a.mode == kModeGlobal ? a.pb.s : a.pb.D; }

// General kernels (sr_grad_fma.cu): every shape and type.
cudaError_t launch_grad_coef_fma(const GradArgs& a);
cudaError_t launch_grad_dict_fma(const GradArgs& a, int* slots);      // partial sums only
// Tensor-core kernels (sr_grad_tc.cu).
bool grad_coef_tc_supported(const GradArgs& a);
bool grad_dict_tc_supported(const GradArgs& a);
cudaError_t launch_grad_coef_tc(const GradArgs& a);
cudaError_t launch_grad_dict_tc(const GradArgs& a, int* slots);       // partial sums only
// Both in one kernel of specialised warps, up to 128 atoms (sr_grad_roles.cu).
bool grad_roles_supported(const GradArgs& a);
cudaError_t launch_grad_roles(const GradArgs& a, int* slots);         // gcoef, and partial sums
// Sums the partial sums of `slots` blocks into gdict and ggamma.
cudaError_t launch_grad_dict_sum(const GradArgs& a, int slots);

struct BalanceArgs {
    const void* coef;
    int coef_dtype;
    const uint8_t* idx;
    const uint8_t* mask;
    float* loss;
    int32_t* counts;
    float* share;
    float* slope;
    void* scratch;
    int n, D, s;
    int64_t HW;
    bool per_frame;
    cudaStream_t st;
};
size_t balance_scratch_bytes(int n, int D, int64_t HW);
cudaError_t launch_balance(const BalanceArgs& a);
cudaError_t launch_balance_grad(const BalanceArgs& a, const float* slope, const float* grad_loss, float weight, void* grad, bool add);

cudaError_t launch_adamw(const sr_adamw_tensor* tensors, int count, int param_dtype, int grad_dtype, int state_bits,
                         const sr_adamw_opts& o, cudaStream_t st);

#ifdef __CUDACC__
// A kernel that sums what the launch before it on the stream wrote: it may be brought up while that one ends (programmatic dependent
// launch) and waits for its end, with all it wrote, in wait_for_launch_before().
// (early = false: an ordinary launch, for a kernel that reads what came before the call without waiting.)
template <typename... Params, typename... Args>
cudaError_t launch_after_smem(void (*kern)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t st, bool early, Args... args)
{
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<Params>(args)...);
}
template <typename... Params, typename... Args>
cudaError_t launch_after(void (*kern)(Params...), dim3 grid, int threads, cudaStream_t st, Args... args)
{
    return launch_after_smem(kern, grid, threads, 0, st, true, args...);
}

// In the launch before: the next one may be brought up now, beside this one (one that depends on nothing this one writes).
__device__ __forceinline__ void let_next_launch_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
#endif

} // namespace sr
