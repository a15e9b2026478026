// Balance loss of a per-pixel selection and its gradient.
//   share p_l(i) = |coef_l(i)| / S(i), S(i) = sum_m |coef_m(i)|;  f_l = counts_l / (s T);  loss = D sum_l f_l mean_i p_l(i)
//   dL/dcoef_l(i) = sign(coef_l) / S(i) (a_l - sum_m a_m p_m(i)),  a_l = D f_l / T (the slope)
//
// Both directions stream the [n][D][H][W] planes once and are bound by that. A block takes a tile of pixels with all its atoms:
// warp w holds atoms w, w + WARPS, ... of the tile in registers (a lane: 8 binary16 or 4 fp32 neighbouring pixels of each,
// one 16-byte load), adds its atoms' magnitudes, and the warps' sums meet in shared memory; then every warp works on from
// its registers, so the planes are read from memory once although a share needs the whole column first.
#include "sr_train.cuh"

namespace sr {

namespace {

constexpr float kSmallestNormal = 1.17549435e-38f;

template <typename CoefT> struct Vec { static constexpr int PX = 16 / (int)sizeof(CoefT); };   // pixels of a lane

// A lane's pixels of one atom, as loaded; widened when used.
template <typename CoefT> struct Piece;
template <> struct Piece<float> {
    float v[4];
    __device__ __forceinline__ void zero() { v[0] = v[1] = v[2] = v[3] = 0.f; }
    __device__ __forceinline__ void load16(const float* p) { const float4 t = __ldcs(reinterpret_cast<const float4*>(p)); v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; }
    __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
    __device__ __forceinline__ float get(int i) const { return v[i]; }
    __device__ __forceinline__ void store16(float* p) const { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Piece<__half> {
    __half2 v[4];
    __device__ __forceinline__ void zero() { v[0] = v[1] = v[2] = v[3] = __half2half2(__ushort_as_half(0)); }
    __device__ __forceinline__ void load16(const __half* p)
    {
        const uint4 t = __ldcs(reinterpret_cast<const uint4*>(p));
        v[0] = *reinterpret_cast<const __half2*>(&t.x); v[1] = *reinterpret_cast<const __half2*>(&t.y);
        v[2] = *reinterpret_cast<const __half2*>(&t.z); v[3] = *reinterpret_cast<const __half2*>(&t.w);
    }
    __device__ __forceinline__ void set(int i, __half x) { v[i / 2] = i % 2 ? __halves2half2(__low2half(v[i / 2]), x) : __halves2half2(x, __high2half(v[i / 2])); }
    __device__ __forceinline__ float get(int i) const { return i % 2 ? __high2float(v[i / 2]) : __low2float(v[i / 2]); }
    __device__ __forceinline__ void store16(__half* p) const
    {
        uint4 t;
        t.x = *reinterpret_cast<const uint32_t*>(&v[0]); t.y = *reinterpret_cast<const uint32_t*>(&v[1]);
        t.z = *reinterpret_cast<const uint32_t*>(&v[2]); t.w = *reinterpret_cast<const uint32_t*>(&v[3]);
        *reinterpret_cast<uint4*>(p) = t;
    }
};
__device__ __forceinline__ float narrow(float v, float*) { return v; }
__device__ __forceinline__ __half narrow(float v, __half*) { return __float2half_rn(v); }

// Pixel of slot i of a lane: neighbouring ones where 16-byte accesses are allowed, else 32 apart (coalesced single elements).
template <int PX, bool VEC> __device__ __forceinline__ int slot_pixel(int lane, int i) { return VEC ? lane * PX + i : lane + 32 * i; }

// The tile's pieces of this warp's atoms.
template <typename CoefT, int AW, int WARPS, bool VEC>
__device__ __forceinline__ void load_pieces(Piece<CoefT> (&x)[AW], const CoefT* frame, int64_t HW, int64_t p0, int D, int warp, int lane)
{
    constexpr int PX = Vec<CoefT>::PX;
#pragma unroll
    for (int a = 0; a < AW; ++a) {
        const int l = warp + a * WARPS;
        x[a].zero();
        if (l < D) {
            const CoefT* src = frame + (int64_t)l * HW + p0;
            if (VEC) {
                if (p0 + lane * PX < HW) x[a].load16(src + lane * PX);
            } else {
#pragma unroll
                for (int i = 0; i < PX; ++i)
                    if (p0 + lane + 32 * i < HW) x[a].set(i, __ldg(src + lane + 32 * i));
            }
        }
    }
}

// ---- forward ---------------------------------------------------------------------------------------------------------------

struct BalanceParams {
    const uint8_t* idx;
    const uint8_t* mask;
    float* part_share;           // [n][bx][D]: sums of shares
    int32_t* part_count;         // [n][bx][D + 1]: counts; last: valid pixels
    unsigned* ticket;            // frames summed so far (balance_sum_kernel)
    int n, D, s, bx;
    int64_t HW;
};

template <typename CoefT, int AW, int WARPS, bool VEC>
__global__ void __launch_bounds__(WARPS * 32)
balance_kernel(const CoefT* __restrict__ coef, const __grid_constant__ BalanceParams p)
{
    constexpr int PX = Vec<CoefT>::PX, TP = 32 * PX, NT = WARPS * 32;
    constexpr int COPIES = 8;                    // of the histogram: fewer threads of a warp meet on a counter
    __shared__ __align__(16) float ssum[WARPS][TP];
    __shared__ int hist[COPIES][257];
    __shared__ int svalid, sempty;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int f = blockIdx.x / p.bx, b = blockIdx.x - f * p.bx;
    const int D = p.D, s = p.s;
    const int64_t HW = p.HW;
    const CoefT* frame = coef + (int64_t)f * D * HW;
    for (int i = tid; i < COPIES * 257; i += NT) (&hist[0][0])[i] = 0;
    if (tid == 0) { svalid = 0; sempty = 0; if (blockIdx.x == 0) *p.ticket = 0u; }
    float total[AW];
#pragma unroll
    for (int a = 0; a < AW; ++a) total[a] = 0.f;
    int valid = 0, empty = 0;                    // pixels that count, and those of them whose sum is too small (their share is 1 / D)
    __syncthreads();
    for (int64_t p0 = (int64_t)b * TP; p0 < HW; p0 += (int64_t)p.bx * TP) {
        Piece<CoefT> x[AW];
        load_pieces<CoefT, AW, WARPS, VEC>(x, frame, HW, p0, D, warp, lane);
        // counts of the listed atoms, a pixel and rank per thread
        for (int i = tid; i < s * TP; i += NT) {
            const int q = i / TP, px = i - q * TP;
            const int64_t at = p0 + px;
            if (at < HW && (!p.mask || __ldg(p.mask + (int64_t)f * HW + at))) {
                const int l = __ldg(p.idx + ((int64_t)f * s + q) * HW + at);
                if (l < D) atomicAdd(&hist[tid % COPIES][l], 1);
            }
        }
        float sum[PX];
#pragma unroll
        for (int i = 0; i < PX; ++i) sum[i] = 0.f;
#pragma unroll
        for (int a = 0; a < AW; ++a)
#pragma unroll
            for (int i = 0; i < PX; ++i) sum[i] += fabsf(x[a].get(i));
#pragma unroll
        for (int i = 0; i < PX; ++i) ssum[warp][slot_pixel<PX, VEC>(lane, i)] = sum[i];
        __syncthreads();
        float r[PX];                             // 1 / S, 0 where the pixel adds nothing here
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            const int px = slot_pixel<PX, VEC>(lane, i);
            const int64_t at = p0 + px;
            float S = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) S += ssum[w][px];
            const bool on = at < HW && (!p.mask || __ldg(p.mask + (int64_t)f * HW + at));
            const bool small = S < kSmallestNormal;
            r[i] = on && !small ? 1.f / S : 0.f;
            if (warp == 0) { valid += on; empty += on && small; }
        }
#pragma unroll
        for (int a = 0; a < AW; ++a)
#pragma unroll
            for (int i = 0; i < PX; ++i) total[a] += r[i] != 0.f ? fabsf(x[a].get(i)) * r[i] : 0.f;   // (a coefficient that does not count may be NaN)
        __syncthreads();
    }
    if (warp == 0) { atomicAdd(&svalid, valid); atomicAdd(&sempty, empty); }
    __syncthreads();
    const int64_t row = (int64_t)blockIdx.x;
#pragma unroll
    for (int a = 0; a < AW; ++a) {
        const int l = warp + a * WARPS;
        float v = total[a];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0 && l < D) p.part_share[row * D + l] = v + (float)sempty / (float)D;
    }
    for (int l = tid; l < D; l += NT) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) c += hist[i][l];
        p.part_count[row * (D + 1) + l] = c;
    }
    if (tid == 0) p.part_count[row * (D + 1) + D] = svalid;
}

struct BalanceSumParams {
    const float* part_share;
    const int32_t* part_count;
    unsigned* ticket;
    double* share_sum;           // [n][D]: sums of shares over a frame
    int32_t* valid;              // [n]
    int32_t* counts;
    float* share;
    float* slope;
    float* loss;
    int n, D, s, bx, per_frame;
};

// Block f adds up frame f (1024 / D threads to an atom, in a fixed order); the block that finishes last then knows every frame's
// sums and writes slopes and loss, frame by frame in their order.
__global__ void __launch_bounds__(1024)
balance_sum_kernel(const __grid_constant__ BalanceSumParams p)
{
    __shared__ double ssum[1024];
    __shared__ int scnt[1024];
    __shared__ int svalid;
    __shared__ bool last;
    const int tid = threadIdx.x, f = blockIdx.x, D = p.D;
    const int groups = 1024 / D, g = tid / D, l = tid - g * D;
    if (tid == 0) svalid = 0;
    __syncthreads();
    double acc = 0.0;
    int c = 0;
    if (g < groups) {
#pragma unroll 8
        for (int b = g; b < p.bx; b += groups) {
            const int64_t row = (int64_t)f * p.bx + b;
            acc += (double)__ldg(p.part_share + row * D + l);
            c += __ldg(p.part_count + row * (D + 1) + l);
        }
    }
    for (int b = tid; b < p.bx; b += 1024) atomicAdd(&svalid, __ldg(p.part_count + ((int64_t)f * p.bx + b) * (D + 1) + D));
    ssum[tid] = acc;
    scnt[tid] = c;
    __syncthreads();
    const int valid = svalid;
    if (tid < D) {
        for (int i = 1; i < groups; ++i) { acc += ssum[i * D + tid]; c += scnt[i * D + tid]; }
        p.share_sum[(int64_t)f * D + tid] = acc;
        p.counts[(int64_t)f * D + tid] = c;
        p.share[(int64_t)f * D + tid] = valid ? (float)(acc / valid) : 0.f;
    }
    if (tid == 0) p.valid[f] = valid;
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // counts of the batch by atom, or each frame's own
    double part = 0.0;
    if (p.per_frame) {
        for (int64_t i = tid; i < (int64_t)p.n * D; i += 1024) {
            const double T = (double)__ldcg(p.valid + i / D);
            const double a = T > 0.0 ? (double)D * __ldcg(p.counts + i) / ((double)p.s * p.n * T * T) : 0.0;
            p.slope[i] = (float)a;
            part += a * __ldcg(p.share_sum + i);
        }
    } else {
        __shared__ double count[256];
        __shared__ double total;
        if (tid == 0) {
            double t = 0.0;
            for (int i = 0; i < p.n; ++i) t += (double)__ldcg(p.valid + i);
            total = t;
        }
        if (tid < D) {
            double t = 0.0;
            for (int i = 0; i < p.n; ++i) t += (double)__ldcg(p.counts + (int64_t)i * D + tid);
            count[tid] = t;
        }
        __syncthreads();
        const double T = total;
        for (int64_t i = tid; i < (int64_t)p.n * D; i += 1024) {
            const double a = T > 0.0 ? (double)D * count[i % D] / ((double)p.s * T * T) : 0.0;
            p.slope[i] = (float)a;
            part += a * __ldcg(p.share_sum + i);
        }
    }
    __syncthreads();
    ssum[tid] = part;
    for (int o = 512; o > 0; o >>= 1) {
        __syncthreads();
        if (tid < o) ssum[tid] += ssum[tid + o];
    }
    if (tid == 0) *p.loss = (float)ssum[0];
}

// ---- backward --------------------------------------------------------------------------------------------------------------

struct BalanceGradParams {
    const uint8_t* mask;
    const float* slope;
    const float* grad_loss;
    float weight;
    int D, tiles;                // tiles of a frame
    int64_t HW;
};

template <typename CoefT, int AW, int WARPS, bool VEC, bool ADD>
__global__ void __launch_bounds__(WARPS * 32)
balance_grad_kernel(const CoefT* __restrict__ coef, CoefT* __restrict__ grad, const __grid_constant__ BalanceGradParams p)
{
    constexpr int PX = Vec<CoefT>::PX, TP = 32 * PX;
    __shared__ __align__(16) float ssum[2][WARPS][TP];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int f = blockIdx.x / p.tiles;
    const int64_t p0 = (int64_t)(blockIdx.x - f * p.tiles) * TP;
    const int D = p.D;
    const int64_t HW = p.HW;
    Piece<CoefT> x[AW];
    load_pieces<CoefT, AW, WARPS, VEC>(x, coef + (int64_t)f * D * HW, HW, p0, D, warp, lane);
    float a[AW];
#pragma unroll
    for (int j = 0; j < AW; ++j) a[j] = warp + j * WARPS < D ? __ldg(p.slope + (int64_t)f * D + warp + j * WARPS) : 0.f;
    float sum[PX], dot[PX];
#pragma unroll
    for (int i = 0; i < PX; ++i) sum[i] = dot[i] = 0.f;
#pragma unroll
    for (int j = 0; j < AW; ++j)
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            const float m = fabsf(x[j].get(i));
            sum[i] += m;
            dot[i] = fmaf(a[j], m, dot[i]);
        }
#pragma unroll
    for (int i = 0; i < PX; ++i) {
        ssum[0][warp][slot_pixel<PX, VEC>(lane, i)] = sum[i];
        ssum[1][warp][slot_pixel<PX, VEC>(lane, i)] = dot[i];
    }
    __syncthreads();
    const float weight = p.grad_loss ? p.weight * __ldg(p.grad_loss) : p.weight;
    float r[PX], mean[PX];
    bool on[PX];
#pragma unroll
    for (int i = 0; i < PX; ++i) {
        const int px = slot_pixel<PX, VEC>(lane, i);
        const int64_t at = p0 + px;
        float S = 0.f, Q = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { S += ssum[0][w][px]; Q += ssum[1][w][px]; }
        on[i] = at < HW && !(S < kSmallestNormal) && (!p.mask || __ldg(p.mask + (int64_t)f * HW + at));
        r[i] = 1.f / S;
        mean[i] = Q * r[i];
    }
#pragma unroll
    for (int j = 0; j < AW; ++j) {
        const int l = warp + j * WARPS;
        if (l >= D) break;
        CoefT* dst = grad + ((int64_t)f * D + l) * HW + p0;
        Piece<CoefT> o;
        o.zero();
        if (VEC && ADD && p0 + lane * PX < HW) o.load16(dst + lane * PX);
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            const float v = x[j].get(i);
            const float d = (a[j] - mean[i]) * weight * r[i];
            const float g = v == 0.f ? 0.f : (v < 0.f ? -d : d);
            if (VEC) {
                if (on[i]) o.set(i, narrow(ADD ? o.get(i) + g : g, (CoefT*)nullptr));
            } else if (p0 + lane + 32 * i < HW) {
                CoefT* d = dst + lane + 32 * i;
                if (ADD) { if (on[i]) *d = narrow((float)*d + g, (CoefT*)nullptr); }
                else *d = narrow(on[i] ? g : 0.f, (CoefT*)nullptr);
            }
        }
        if (VEC && p0 + lane * PX < HW) o.store16(dst + lane * PX);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

int pixels_of_tile(int coef_dtype) { return coef_dtype == SR_F16 ? 256 : 128; }

// Blocks of a frame. Four blocks a multiprocessor over all frames, but no more than tiles.
int frame_blocks(int n, int64_t HW, int coef_dtype)
{
    const int64_t tiles = (HW + pixels_of_tile(coef_dtype) - 1) / pixels_of_tile(coef_dtype);
    int64_t want = (4ll * sm_count() + n - 1) / n;
    if (want < 1) want = 1;
    return (int)(want < tiles ? want : tiles);
}

// Scratch: share sums [n][D] fp64, partial shares, partial counts, valid pixels [n], the ticket.
struct Scratch { double* share_sum; float* part_share; int32_t* part_count; int32_t* valid; unsigned* ticket; size_t bytes; };
Scratch carve(void* base, int n, int D, int bx)
{
    uint8_t* p = static_cast<uint8_t*>(base);
    auto take = [&](size_t bytes) { uint8_t* at = p; p += (bytes + 15) & ~(size_t)15; return at; };
    Scratch s;
    s.share_sum = (double*)take((size_t)n * D * 8);
    s.part_share = (float*)take((size_t)n * bx * D * 4);
    s.part_count = (int32_t*)take((size_t)n * bx * (D + 1) * 4);
    s.valid = (int32_t*)take((size_t)n * 4);
    s.ticket = (unsigned*)take(4);
    s.bytes = (size_t)(p - static_cast<uint8_t*>(base));
    return s;
}

template <typename CoefT, int AW, int WARPS>
cudaError_t forward_t(const BalanceArgs& a, const BalanceParams& p, bool vec)
{
    const unsigned blocks = (unsigned)(a.n * p.bx);
    if (vec) balance_kernel<CoefT, AW, WARPS, true><<<blocks, WARPS * 32, 0, a.st>>>((const CoefT*)a.coef, p);
    else balance_kernel<CoefT, AW, WARPS, false><<<blocks, WARPS * 32, 0, a.st>>>((const CoefT*)a.coef, p);
    return cudaGetLastError();
}

template <typename CoefT, int AW, int WARPS>
cudaError_t backward_t(const BalanceArgs& a, const BalanceGradParams& p, void* grad, bool vec, bool add)
{
    const unsigned blocks = (unsigned)(a.n * p.tiles);
    const CoefT* c = (const CoefT*)a.coef;
    CoefT* g = (CoefT*)grad;
    if (vec && add) balance_grad_kernel<CoefT, AW, WARPS, true, true><<<blocks, WARPS * 32, 0, a.st>>>(c, g, p);
    else if (vec) balance_grad_kernel<CoefT, AW, WARPS, true, false><<<blocks, WARPS * 32, 0, a.st>>>(c, g, p);
    else if (add) balance_grad_kernel<CoefT, AW, WARPS, false, true><<<blocks, WARPS * 32, 0, a.st>>>(c, g, p);
    else balance_grad_kernel<CoefT, AW, WARPS, false, false><<<blocks, WARPS * 32, 0, a.st>>>(c, g, p);
    return cudaGetLastError();
}

// Atoms of a warp (registers) and warps of a block by D.
#define SR_BALANCE_BY_ATOMS(D, call)                                   \
    ((D) <= 16 ? call(2, 8) : (D) <= 32 ? call(4, 8) : (D) <= 48 ? call(6, 8) : (D) <= 80 ? call(10, 8) : (D) <= 128 ? call(8, 16) : call(16, 16))

template <typename CoefT> cudaError_t forward(const BalanceArgs& a, const BalanceParams& p, bool vec)
{
#define SR_CALL(AW, WARPS) forward_t<CoefT, AW, WARPS>(a, p, vec)
    return SR_BALANCE_BY_ATOMS(a.D, SR_CALL);
#undef SR_CALL
}

template <typename CoefT> cudaError_t backward(const BalanceArgs& a, const BalanceGradParams& p, void* grad, bool vec, bool add)
{
#define SR_CALL(AW, WARPS) backward_t<CoefT, AW, WARPS>(a, p, grad, vec, add)
    return SR_BALANCE_BY_ATOMS(a.D, SR_CALL);
#undef SR_CALL
}

bool vectors(const BalanceArgs& a, const void* other)
{
    return (((uintptr_t)a.coef | (uintptr_t)other) & 15) == 0 && a.HW % (a.coef_dtype == SR_F16 ? 8 : 4) == 0;
}

} // namespace

size_t balance_scratch_bytes(int n, int D, int64_t HW)
{
    // (fp32 tiles are the smaller ones, so its blocks are never fewer)
    return carve(nullptr, n, D, frame_blocks(n, HW, SR_F32)).bytes;
}

cudaError_t launch_balance(const BalanceArgs& a)
{
    const int bx = frame_blocks(a.n, a.HW, a.coef_dtype);
    if ((int64_t)a.n * bx > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const Scratch sc = carve(a.scratch, a.n, a.D, bx);
    const BalanceParams p{a.idx, a.mask, sc.part_share, sc.part_count, sc.ticket, a.n, a.D, a.s, bx, a.HW};
    const bool vec = vectors(a, nullptr);
    if (cudaError_t e = a.coef_dtype == SR_F16 ? forward<__half>(a, p, vec) : forward<float>(a, p, vec)) return e;
    const BalanceSumParams q{sc.part_share, sc.part_count, sc.ticket, sc.share_sum, sc.valid, a.counts, a.share, a.slope, a.loss,
                             a.n, a.D, a.s, bx, a.per_frame ? 1 : 0};
    balance_sum_kernel<<<a.n, 1024, 0, a.st>>>(q);
    count_launches(2);
    return cudaGetLastError();
}

cudaError_t launch_balance_grad(const BalanceArgs& a, const float* slope, const float* grad_loss, float weight, void* grad, bool add)
{
    const int64_t tiles = (a.HW + pixels_of_tile(a.coef_dtype) - 1) / pixels_of_tile(a.coef_dtype);
    if (tiles * a.n > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const BalanceGradParams p{a.mask, slope, grad_loss, weight, a.D, (int)tiles, a.HW};
    const bool vec = vectors(a, grad);
    count_launches(1);
    return a.coef_dtype == SR_F16 ? backward<__half>(a, p, grad, vec, add) : backward<float>(a, p, grad, vec, add);
}

} // namespace sr
