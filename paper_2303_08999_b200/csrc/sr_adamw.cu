// AdamW over many tensors in few launches. Bound by memory: a step reads p, g, m, v and writes p, m, v once (fp32: 28 bytes an
// element; 8-bit states 16).
//
// The tensors travel as kernel arguments (up to kTensors of them a launch), so the call copies no table and can be captured.
// A block takes a run of kRun elements of one tensor, found by bisection over the tensors' first blocks; with 8-bit states a warp
// takes 256 elements, eight a lane, at a time, which is the unit of one scale: the two largest magnitudes are a warp's shuffles.
#include <math.h>

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "sr_train.cuh"

namespace sr {

namespace {

constexpr int kTensors = 440;                 // 440 x 61 bytes + the rest stay below the 32764 bytes of kernel arguments
constexpr int kFewTensors = 16;               // a short list is a short launch: three tensors 12.3 -> 9.3 us
constexpr int kUnit = 256, kRun = 2048;       // elements of a scale; of a block (eight warps, one unit each)
constexpr float kPerF8Max = 1.f / 448.f;      // (a product instead of a quotient: as PyTorch divides by a number on the GPU)

template <int N> struct AdamwList {
    void* param[N];
    const void* grad[N];
    void* m[N];
    void* v[N];
    float* m_scale[N];
    float* v_scale[N];
    int64_t n[N];
    int first[N + 1];                         // first block of each tensor
    uint8_t wide[N];                          // 16-byte accesses allowed
    int count;
};

struct AdamwScalars {
    float beta1, beta2, one_beta1, one_beta2, eps, decay, grad_scale;      // decay: weight_decay
    float lr, correct1, correct2;             // correct1 = 1 / (1 - beta1^t), correct2 = 1 / sqrt(1 - beta2^t)
    float log_beta1, log_beta2;               // for a step count on the device
    const float* lr_dev;
    const int64_t* step_dev;
    const int32_t* skip_dev;
};

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T narrow_to(float v);
template <> __device__ __forceinline__ float narrow_to<float>(float v) { return v; }
template <> __device__ __forceinline__ __half narrow_to<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// N neighbouring elements, in 16-byte (or, of N narrow ones, whole) accesses.
template <typename T, int N> struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Pack { T v[N]; };

template <typename T, int N> __device__ __forceinline__ void read(float (&out)[N], const T* p, bool wide, int have)
{
    if (wide && have >= N) {
        const Pack<T, N> t = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = widen(t.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = i < have ? widen(p[i]) : 0.f;
    }
}
template <typename T, int N> __device__ __forceinline__ void write(T* p, const float (&in)[N], bool wide, int have)
{
    if (wide && have >= N) {
        Pack<T, N> t;
#pragma unroll
        for (int i = 0; i < N; ++i) t.v[i] = narrow_to<T>(in[i]);
        *reinterpret_cast<Pack<T, N>*>(p) = t;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) p[i] = narrow_to<T>(in[i]);
    }
}

// Eight e4m3 codes as values; eight values to codes, rounded to nearest even, beyond 448 held there.
__device__ __forceinline__ void e4m3_values(float (&out)[8], const uint8_t* codes)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(*reinterpret_cast<const __nv_fp8x2_storage_t*>(codes + i), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        out[i] = f.x;
        out[i + 1] = f.y;
    }
}
__device__ __forceinline__ void e4m3_codes(uint8_t* codes, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i += 2)
        *reinterpret_cast<__nv_fp8x2_storage_t*>(codes + i) = __nv_cvt_float2_to_fp8x2(make_float2(v[i], v[i + 1]), __NV_SATFINITE, __NV_E4M3);
}

// v / scale for a block, each quotient rounded once, so that a code is the quotient's, ties and all. Markstein's correction (IBM J. Res.
// Dev. 34, 1990): q = v r, with r the rounded reciprocal, may be a unit off; its remainder v - q scale is exact, and q + remainder r rounds
// to the quotient. A division where the remainder or r could leave the normal numbers.
__device__ __forceinline__ void over_scale(float (&out)[8], const float (&v)[8], float scale)
{
    if (scale >= 7.8886091e-31f && scale <= 1.2676506e30f) {          // 2^-100, 2^100
        const float inv = 1.f / scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q = v[i] * inv;
            out[i] = fmaf(fmaf(-q, scale, v[i]), inv, q);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = scale > 0.f ? v[i] / scale : 0.f;
    }
}

// A parameter's step takes division, and with 32-bit states the root, at the speed of their approximate instructions (2 and 1 units in the
// last place of the step, which is small beside the parameter). Exact ones, 63 M parameters: fp32 262 us both ways; 16-bit parameters
// and gradients 207 -> 229; 8-bit states 12 more; three small tensors 9.2 -> 11.3. The 8-bit states' root is exact: it is stored.
__device__ __forceinline__ float fast_sqrt(float v)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The larger one, NaN where either is: a block with a value that is not finite has a scale that is not, and so no state that looks valid.
__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max_or_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

template <typename P, typename G, int BITS, int N>
__global__ void __launch_bounds__(256)
adamw_kernel(const __grid_constant__ AdamwList<N> list, const __grid_constant__ AdamwScalars o)
{
    if (o.skip_dev && __ldg(o.skip_dev) != 0) return;
    const int block = blockIdx.x;
    int lo = 0, hi = list.count;              // first[lo] <= block < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (list.first[mid] <= block) lo = mid;
        else hi = mid;
    }
    const int64_t n = list.n[lo];
    const bool wide = list.wide[lo] != 0;
    const int64_t unit = (int64_t)(block - list.first[lo]) * (kRun / kUnit) + threadIdx.x / 32;
    const int64_t at = unit * kUnit + (threadIdx.x % 32) * 8;
    if (unit * kUnit >= n) return;            // whole warps
    const int have = (int)(n - at < 8 ? (n - at > 0 ? n - at : 0) : 8);

    float lr = o.lr, c1 = o.correct1, c2 = o.correct2;
    if (o.lr_dev) lr = __ldg(o.lr_dev);
    if (o.step_dev) {                         // 1 - beta^t = -expm1(t ln beta), exact to a few units for every t
        const float t = (float)__ldg(o.step_dev);
        c1 = -1.f / expm1f(t * o.log_beta1);
        c2 = rsqrtf(-expm1f(t * o.log_beta2));
    }
    const float keep = 1.f - lr * o.decay, rate = lr * c1;

    P* pp = static_cast<P*>(list.param[lo]) + at;
    const G* pg = static_cast<const G*>(list.grad[lo]) + at;
    float p[8], g[8], m[8], v[8];
    read<P, 8>(p, pp, wide, have);
    read<G, 8>(g, pg, wide, have);
    if (BITS == 32) {
        read<float, 8>(m, static_cast<const float*>(list.m[lo]) + at, wide, have);
        read<float, 8>(v, static_cast<const float*>(list.v[lo]) + at, wide, have);
    } else {
        const uint8_t* cm = static_cast<const uint8_t*>(list.m[lo]) + at;
        const uint8_t* cv = static_cast<const uint8_t*>(list.v[lo]) + at;
        const float sm = list.m_scale[lo][unit], sv = list.v_scale[lo][unit];
        alignas(8) uint8_t a[8], b[8];
        if (wide && have == 8) {
            *reinterpret_cast<uint2*>(a) = *reinterpret_cast<const uint2*>(cm);
            *reinterpret_cast<uint2*>(b) = *reinterpret_cast<const uint2*>(cv);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) { a[i] = i < have ? cm[i] : 0; b[i] = i < have ? cv[i] : 0; }
        }
        e4m3_values(m, a);
        e4m3_values(v, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] *= sm;
            const float root = sv * v[i];
            v[i] = root * root;
        }
    }
    float root[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = g[i] * o.grad_scale;
        if (BITS == 8) {
            // Every operation rounded by itself: where a sum is contracted, a value next to the middle of two codes goes to the other one
            // (8 of 5 M). With the exact root and quotients: 63 M parameters 174 -> 188 us.
            m[i] = __fadd_rn(__fmul_rn(o.beta1, m[i]), __fmul_rn(o.one_beta1, gi));
            v[i] = __fadd_rn(__fmul_rn(o.beta2, v[i]), __fmul_rn(o.one_beta2, __fmul_rn(gi, gi)));
            root[i] = __fsqrt_rn(v[i]);
        } else {
            m[i] = fmaf(o.beta1, m[i], o.one_beta1 * gi);
            v[i] = fmaf(o.beta2, v[i], o.one_beta2 * (gi * gi));
            root[i] = fast_sqrt(v[i]);
        }
        p[i] = fmaf(p[i], keep, -__fdividef(rate * m[i], fmaf(root[i], c2, o.eps)));
    }
    write<P, 8>(pp, p, wide, have);
    if (BITS == 32) {
        write<float, 8>(static_cast<float*>(list.m[lo]) + at, m, wide, have);
        write<float, 8>(static_cast<float*>(list.v[lo]) + at, v, wide, have);
    } else {
        float top_m = 0.f, top_v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) { top_m = max_or_nan(top_m, fabsf(m[i])); top_v = max_or_nan(top_v, root[i]); }
        const float sm = warp_max(top_m) * kPerF8Max, sv = warp_max(top_v) * kPerF8Max;
        alignas(8) uint8_t a[8], b[8];
        float q[8];
        over_scale(q, m, sm);
        e4m3_codes(a, q);
        over_scale(q, root, sv);
#pragma unroll
        for (int i = 0; i < 8; ++i)                                   // (a root that is not zero is held as the smallest code at least:
            if (root[i] > 0.f && sv > 0.f && q[i] < 0.001953125f) q[i] = 0.001953125f;      // the next step divides by it)
        e4m3_codes(b, q);
        uint8_t* cm = static_cast<uint8_t*>(list.m[lo]) + at;
        uint8_t* cv = static_cast<uint8_t*>(list.v[lo]) + at;
        if (wide && have == 8) {
            *reinterpret_cast<uint2*>(cm) = *reinterpret_cast<const uint2*>(a);
            *reinterpret_cast<uint2*>(cv) = *reinterpret_cast<const uint2*>(b);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) { cm[i] = a[i]; cv[i] = b[i]; }
        }
        if (threadIdx.x % 32 == 0) { list.m_scale[lo][unit] = sm; list.v_scale[lo][unit] = sv; }
    }
}

struct Launch { const AdamwScalars& o; int param_dtype, grad_dtype, bits, blocks; cudaStream_t st; };

template <typename P, typename G, int N> void launch_pg(const AdamwList<N>& list, const Launch& l)
{
    if (l.bits == 8) adamw_kernel<P, G, 8, N><<<l.blocks, 256, 0, l.st>>>(list, l.o);
    else adamw_kernel<P, G, 32, N><<<l.blocks, 256, 0, l.st>>>(list, l.o);
}

template <typename P, int N> void launch_p(const AdamwList<N>& list, const Launch& l)
{
    switch (l.grad_dtype) {
    case SR_F16: return launch_pg<P, __half, N>(list, l);
    case SR_BF16: return launch_pg<P, __nv_bfloat16, N>(list, l);
    default: return launch_pg<P, float, N>(list, l);
    }
}

// Launches of up to N tensors each.
template <int N> cudaError_t launch_lists(const sr_adamw_tensor* tensors, int count, Launch l)
{
    AdamwList<N> list;                        // (only the entries in use are read)
    int i = 0;
    while (i < count) {
        int64_t blocks = 0;
        list.count = 0;
        for (; i < count && list.count < N; ++i) {
            const sr_adamw_tensor& x = tensors[i];
            if (x.n == 0) continue;
            const int64_t more = (x.n + kRun - 1) / kRun;
            if (more > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
            if (blocks + more > 0x7FFFFFFF) break;
            const int k = list.count++;
            list.param[k] = x.param; list.grad[k] = x.grad; list.m[k] = x.m; list.v[k] = x.v;
            list.m_scale[k] = x.m_scale; list.v_scale[k] = x.v_scale; list.n[k] = x.n;
            list.first[k] = (int)blocks;
            list.wide[k] = (((uintptr_t)x.param | (uintptr_t)x.grad | (uintptr_t)x.m | (uintptr_t)x.v) & 15) == 0;
            blocks += more;
        }
        if (!list.count) break;
        list.first[list.count] = (int)blocks;
        l.blocks = (int)blocks;
        switch (l.param_dtype) {
        case SR_F16: launch_p<__half, N>(list, l); break;
        case SR_BF16: launch_p<__nv_bfloat16, N>(list, l); break;
        default: launch_p<float, N>(list, l);
        }
        count_launches(1);
        if (cudaError_t e = cudaGetLastError()) return e;
    }
    return cudaSuccess;
}

} // namespace

cudaError_t launch_adamw(const sr_adamw_tensor* tensors, int count, int param_dtype, int grad_dtype, int state_bits,
                         const sr_adamw_opts& o, cudaStream_t st)
{
    AdamwScalars sc{};
    sc.beta1 = (float)o.beta1; sc.beta2 = (float)o.beta2;
    sc.one_beta1 = (float)(1.0 - o.beta1); sc.one_beta2 = (float)(1.0 - o.beta2);
    sc.eps = (float)o.eps; sc.decay = (float)o.weight_decay; sc.grad_scale = (float)o.grad_scale; sc.lr = (float)o.lr;
    const double t = (double)o.step;
    sc.correct1 = (float)(1.0 / (1.0 - pow(o.beta1, t)));
    sc.correct2 = (float)(1.0 / sqrt(1.0 - pow(o.beta2, t)));
    sc.log_beta1 = (float)log(o.beta1); sc.log_beta2 = (float)log(o.beta2);
    sc.lr_dev = o.lr_dev; sc.step_dev = o.step_dev; sc.skip_dev = o.skip_dev;
    const Launch l{sc, param_dtype, grad_dtype, state_bits, 0, st};
    return count <= kFewTensors ? launch_lists<kFewTensors>(tensors, count, l) : launch_lists<kTensors>(tensors, count, l);
}

} // namespace sr
