// Balance loss of a per-pixel selection and its gradient.
//   share p_l(i) = |coef_l(i)| / S(i), S(i) = sum_m |coef_m(i)|;  f_l = counts_l / (s T);  loss = D sum_l f_l mean_i p_l(i)
//   dL/dcoef_l(i) = sign(coef_l) / S(i) (a_l - sum_m a_m p_m(i)),  a_l = D f_l / T (the slope)
//
// Both directions stream the [n][D][H][W] planes once and are bound by that. A block takes a tile of 256 (binary16) or 128 (fp32)
// pixels with all its atoms: warp w holds atoms w, w + WARPS, ... of the tile in registers, as loaded (a lane: 16 bytes of each), and adds
// their magnitudes; the warps' sums meet in shared memory, where one thread a pixel finishes them; then every warp works on from its
// registers, so the planes are read from memory once although a share needs the whole column first. Widening costs an instruction
// an element, so magnitudes and signs are taken on the packed words.
#include <type_traits>

#include "sr_train.cuh"

namespace sr {

namespace {

constexpr float kSmallestNormal = 1.17549435e-38f;

// A lane's share of one atom of a tile: four 32-bit words. VEC: neighbouring pixels, one 16-byte access (planes and bases that allow it); else the words' elements are 32 pixels apart, so that single-element accesses of a warp are one run.
template <typename CoefT> struct Lane;
template <> struct Lane<float> {
    static constexpr int PER = 1;                // pixels of a word
    static constexpr uint32_t kMagnitude = 0x7FFFFFFFu;
    static __device__ __forceinline__ float get(const uint32_t* v, int i) { return __uint_as_float(v[i]); }
    static __device__ __forceinline__ float add(const uint32_t* v, int i, float s) { return s + __uint_as_float(v[i]); }
    static __device__ __forceinline__ uint32_t one(const float* p) { return __float_as_uint(__ldcs(p)); }
    static __device__ __forceinline__ void put(uint32_t* v, int i, uint32_t x) { v[i] = x; }
    static __device__ __forceinline__ uint32_t keep(const bool* on, int j) { return on[j] ? kMagnitude : 0u; }
};
template <> struct Lane<__half> {
    static constexpr int PER = 2;
    static constexpr uint32_t kMagnitude = 0x7FFF7FFFu;
    static __device__ __forceinline__ float get(const uint32_t* v, int i)
    {
        const __half2 h = *reinterpret_cast<const __half2*>(&v[i / 2]);
        return i % 2 ? __high2float(h) : __low2float(h);
    }
    // s + element i: the addition that takes a binary16 operand
    static __device__ __forceinline__ float add(const uint32_t* v, int i, float s)
    {
        float d;
        if (i % 2) asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tadd.f32.f16 %0, b, %2;\n\t}" : "=f"(d) : "r"(v[i / 2]), "f"(s));
        else asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tadd.f32.f16 %0, a, %2;\n\t}" : "=f"(d) : "r"(v[i / 2]), "f"(s));
        return d;
    }
    static __device__ __forceinline__ uint32_t one(const __half* p) { return (uint32_t)__half_as_ushort(__ldcs(p)); }
    static __device__ __forceinline__ void put(uint32_t* v, int i, uint32_t x) { v[i / 2] = i % 2 ? __byte_perm(v[i / 2], x, 0x5410) : x; }
    static __device__ __forceinline__ uint32_t keep(const bool* on, int j) { return (on[2 * j] ? 0x7FFFu : 0u) | (on[2 * j + 1] ? 0x7FFF0000u : 0u); }
};

template <int PX, bool VEC> __device__ __forceinline__ int slot_pixel(int lane, int i) { return VEC ? lane * PX + i : lane + 32 * i; }

constexpr int NW = 4;                            // words of a lane
__device__ __forceinline__ void unpack(uint32_t* x, const uint4& t) { x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w; }

// The tile's words of this warp's atoms; zero beyond the frame's end.
template <typename CoefT, int AW, int WARPS, bool VEC>
__device__ __forceinline__ void load_words(uint32_t (&x)[AW][NW], const CoefT* tile, int64_t HW, int left, int D, int warp, int lane)
{
    using L = Lane<CoefT>;
    constexpr int PX = NW * L::PER;
    const CoefT* src = tile + (int64_t)warp * HW + (VEC ? lane * PX : lane);
    const bool whole = left >= 32 * PX;
#pragma unroll
    for (int a = 0; a < AW; ++a, src += WARPS * HW) {
#pragma unroll
        for (int j = 0; j < NW; ++j) x[a][j] = 0u;
        if (warp + a * WARPS < D) {
            if (VEC) {
                if (lane * PX < left) unpack(x[a], __ldcs(reinterpret_cast<const uint4*>(src)));
            } else if (whole) {
#pragma unroll
                for (int i = 0; i < PX; ++i) L::put(x[a], i, L::one(src + 32 * i));
            } else {
#pragma unroll
                for (int i = 0; i < PX; ++i) L::put(x[a], i, lane + 32 * i < left ? L::one(src + 32 * i) : 0u);
            }
        }
    }
}

// What to keep of each word: its magnitude bits, nothing of pixels that do not count (whatever stands there).
template <typename CoefT, bool VEC>
__device__ __forceinline__ void keep_words(uint32_t (&keep)[NW], const uint8_t* mask, int left, int lane)
{
    using L = Lane<CoefT>;
    constexpr int PX = NW * L::PER;
#pragma unroll
    for (int j = 0; j < NW; ++j) keep[j] = L::kMagnitude;
    if (mask) {
        bool on[PX];
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            const int px = slot_pixel<PX, VEC>(lane, i);
            on[i] = px < left && __ldg(mask + px) != 0;
        }
#pragma unroll
        for (int j = 0; j < NW; ++j) keep[j] = L::keep(on, j);
    }
}

template <int PX, bool VEC> __device__ __forceinline__ void put_pixels(float* row, const float (&v)[PX], int lane)
{
    if (VEC && PX % 4 == 0) {
#pragma unroll
        for (int j = 0; j < PX / 4; ++j) *reinterpret_cast<float4*>(row + lane * PX + 4 * j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    } else if (VEC) {
#pragma unroll
        for (int j = 0; j < PX / 2; ++j) *reinterpret_cast<float2*>(row + lane * PX + 2 * j) = make_float2(v[2 * j], v[2 * j + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < PX; ++i) row[lane + 32 * i] = v[i];
    }
}
template <int PX, bool VEC> __device__ __forceinline__ void get_pixels(float (&v)[PX], const float* row, int lane)
{
    if (VEC && PX % 4 == 0) {
#pragma unroll
        for (int j = 0; j < PX / 4; ++j) {
            const float4 t = *reinterpret_cast<const float4*>(row + lane * PX + 4 * j);
            v[4 * j] = t.x; v[4 * j + 1] = t.y; v[4 * j + 2] = t.z; v[4 * j + 3] = t.w;
        }
    } else if (VEC) {
#pragma unroll
        for (int j = 0; j < PX / 2; ++j) {
            const float2 t = *reinterpret_cast<const float2*>(row + lane * PX + 2 * j);
            v[2 * j] = t.x; v[2 * j + 1] = t.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PX; ++i) v[i] = row[lane + 32 * i];
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

// Threads of a multiprocessor that leave each the registers for its words and what it does with them.
constexpr int resident_threads(int words) { return words <= 24 ? 1024 : words <= 36 ? 768 : 512; }

template <typename CoefT, int AW, int WARPS, bool VEC>
__global__ void __launch_bounds__(WARPS * 32, resident_threads(AW * NW) / (WARPS * 32))
balance_kernel(const CoefT* __restrict__ coef, const __grid_constant__ BalanceParams p)
{
    using L = Lane<CoefT>;
    constexpr int PX = NW * L::PER, TP = 32 * PX, NT = WARPS * 32, RANKS = NT / TP;   // threads a pixel
    constexpr int COPIES = 8;                    // of the histogram: fewer threads of a warp meet on a counter
    __shared__ __align__(16) float ssum[WARPS][TP];
    __shared__ __align__(16) float sr[TP];
    __shared__ int hist[COPIES][257];
    __shared__ int svalid, sempty;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int f = blockIdx.x / p.bx, b = blockIdx.x - f * p.bx;
    const int D = p.D, s = p.s, px = tid % TP, rank0 = tid / TP;
    const int64_t HW = p.HW;
    const CoefT* frame = coef + (int64_t)f * D * HW;
    const uint8_t* frame_idx = p.idx + (int64_t)f * s * HW;
    const uint8_t* frame_mask = p.mask ? p.mask + (int64_t)f * HW : nullptr;
    for (int i = tid; i < COPIES * 257; i += NT) (&hist[0][0])[i] = 0;
    if (tid == 0) { svalid = 0; sempty = 0; if (blockIdx.x == 0) *p.ticket = 0u; }
    float total[AW];
#pragma unroll
    for (int a = 0; a < AW; ++a) total[a] = 0.f;
    int valid = 0, empty = 0;                    // pixels that count, and those of them whose sum is too small (their share is 1 / D)
    __syncthreads();
    for (int64_t p0 = (int64_t)b * TP; p0 < HW; p0 += (int64_t)p.bx * TP) {
        const int left = (int)min((int64_t)TP, HW - p0);
        uint32_t x[AW][NW], keep[NW];
        load_words<CoefT, AW, WARPS, VEC>(x, frame + p0, HW, left, D, warp, lane);
        const bool on = px < left && (!frame_mask || __ldg(frame_mask + p0 + px) != 0);
        if (on) {                                // counts of the listed atoms
            const uint8_t* at = frame_idx + (int64_t)rank0 * HW + p0 + px;
            int q = rank0;
            for (; q + 3 * RANKS < s; q += 4 * RANKS) {
                int l[4];
#pragma unroll
                for (int i = 0; i < 4; ++i, at += RANKS * HW) l[i] = __ldcs(at);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (l[i] < D) atomicAdd(&hist[lane % COPIES][l[i]], 1);
            }
            for (; q < s; q += RANKS, at += RANKS * HW) {
                const int l = __ldcs(at);
                if (l < D) atomicAdd(&hist[lane % COPIES][l], 1);
            }
        }
        keep_words<CoefT, VEC>(keep, frame_mask ? frame_mask + p0 : nullptr, left, lane);
        float sum[PX];
#pragma unroll
        for (int i = 0; i < PX; ++i) sum[i] = 0.f;
#pragma unroll
        for (int a = 0; a < AW; ++a) {
#pragma unroll
            for (int j = 0; j < NW; ++j) x[a][j] &= keep[j];
#pragma unroll
            for (int i = 0; i < PX; ++i) sum[i] = L::add(x[a], i, sum[i]);
        }
        put_pixels<PX, VEC>(ssum[warp], sum, lane);
        __syncthreads();
        if (tid < TP) {
            float S = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) S += ssum[w][px];
            const bool small = S < kSmallestNormal;
            sr[px] = on && !small ? 1.f / S : 0.f;
            valid += on;
            empty += on && small;
        }
        __syncthreads();
        float r[PX];
        get_pixels<PX, VEC>(r, sr, lane);
#pragma unroll
        for (int a = 0; a < AW; ++a)
#pragma unroll
            for (int i = 0; i < PX; ++i) total[a] = fmaf(L::get(x[a], i), r[i], total[a]);
    }
    if (tid < TP) {
        valid = __reduce_add_sync(0xffffffffu, valid);
        empty = __reduce_add_sync(0xffffffffu, empty);
        if (lane == 0) { atomicAdd(&svalid, valid); atomicAdd(&sempty, empty); }
    }
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

// Block (frame f, atoms 8 a .. 8 a + 7) adds up the frame's partial sums: 32 threads to an atom, first within a warp, then over the
// eight warps in order; the block that finishes last then knows every frame's sums and writes slopes and loss.
constexpr int kSumAtoms = 8, kSumThreads = 256;
__global__ void __launch_bounds__(kSumThreads)
balance_sum_kernel(const __grid_constant__ BalanceSumParams p)
{
    __shared__ double ssum[kSumThreads / 32][kSumAtoms];
    __shared__ int scnt[kSumThreads / 32][kSumAtoms], svalid[kSumThreads / 32];
    __shared__ bool last;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, f = blockIdx.x, D = p.D;
    const int i8 = tid % kSumAtoms, g = tid / kSumAtoms, l = blockIdx.y * kSumAtoms + i8;
    wait_for_launch_before();
    double acc = 0.0;
    int c = 0, v = 0;
    const float* ps = p.part_share + (int64_t)f * p.bx * D + min(l, D - 1);
    const int32_t* pc = p.part_count + (int64_t)f * p.bx * (D + 1);
#pragma unroll 8
    for (int b = g; b < p.bx; b += kSumThreads / kSumAtoms) {
        acc += (double)__ldg(ps + (int64_t)b * D);
        c += __ldg(pc + (int64_t)b * (D + 1) + min(l, D - 1));
        if (i8 == 0) v += __ldg(pc + (int64_t)b * (D + 1) + D);
    }
#pragma unroll
    for (int o = 16; o >= kSumAtoms; o >>= 1) {
        acc += __shfl_xor_sync(0xffffffffu, acc, o);
        c += __shfl_xor_sync(0xffffffffu, c, o);
    }
    v = __reduce_add_sync(0xffffffffu, v);
    if (lane < kSumAtoms) { ssum[warp][lane] = acc; scnt[warp][lane] = c; }
    if (lane == 0) svalid[warp] = v;
    __syncthreads();
    int valid = 0;
#pragma unroll
    for (int w = 0; w < kSumThreads / 32; ++w) valid += svalid[w];
    if (tid < kSumAtoms && l < D) {
        for (int w = 1; w < kSumThreads / 32; ++w) { acc += ssum[w][tid]; c += scnt[w][tid]; }
        p.share_sum[(int64_t)f * D + l] = acc;
        p.counts[(int64_t)f * D + l] = c;
        p.share[(int64_t)f * D + l] = valid ? (float)(acc / valid) : 0.f;
    }
    if (tid == 0 && blockIdx.y == 0) p.valid[f] = valid;
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(p.ticket, 1u) == gridDim.x * gridDim.y - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // counts of the batch by atom, or each frame's own
    double part = 0.0;
    if (p.per_frame) {
        for (int64_t i = tid; i < (int64_t)p.n * D; i += kSumThreads) {
            const double T = (double)__ldcg(p.valid + i / D);
            const double a = T > 0.0 ? (double)D * __ldcg(p.counts + i) / ((double)p.s * p.n * T * T) : 0.0;
            p.slope[i] = (float)a;
            part += a * __ldcg(p.share_sum + i);
        }
    } else {
        __shared__ double count[256];
        double T = 0.0;
        for (int i = 0; i < p.n; ++i) T += (double)__ldcg(p.valid + i);
        if (tid < D) {
            double t = 0.0;
            for (int i = 0; i < p.n; ++i) t += (double)__ldcg(p.counts + (int64_t)i * D + tid);
            count[tid] = T > 0.0 ? (double)D * t / ((double)p.s * T * T) : 0.0;
        }
        __syncthreads();
        for (int64_t i = tid; i < (int64_t)p.n * D; i += kSumThreads) {
            const double a = count[i % D];
            p.slope[i] = (float)a;
            part += a * __ldcg(p.share_sum + i);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    __syncthreads();
    if (lane == 0) ssum[warp][0] = part;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kSumThreads / 32; ++w) part += ssum[w][0];
        *p.loss = (float)part;
    }
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

// The results of a word: the factors d of the magnitudes with the coefficients' signs, zero where a coefficient is; or those added to
// the word `old`. (A NaN in a pixel that does not count meets d = 0.)
template <bool ADD> __device__ __forceinline__ uint32_t result_word(const float*, uint32_t x, uint32_t old, const float* d)
{
    const float g = __uint_as_float(x) == 0.f ? 0.f : __uint_as_float(__float_as_uint(d[0]) ^ (x & 0x80000000u));
    return __float_as_uint(ADD ? __uint_as_float(old) + g : g);
}
template <bool ADD> __device__ __forceinline__ uint32_t result_word(const __half*, uint32_t x, uint32_t old, const float* d)
{
    const uint32_t some = __hne2_mask(*reinterpret_cast<const __half2*>(&x), __half2half2(__ushort_as_half(0)));
    if (!ADD) {                                  // rounding is symmetric: the sign may come after it
        const __half2 g = __floats2half2_rn(d[0], d[1]);
        return (*reinterpret_cast<const uint32_t*>(&g) ^ (x & 0x80008000u)) & some;
    }
    const uint32_t sign = ((x & 0x80008000u) | 0x3C003C00u) & some;              // +1, -1 or 0 each
    const __half2 sg = *reinterpret_cast<const __half2*>(&sign), o = *reinterpret_cast<const __half2*>(&old);
    const __half2 g = __floats2half2_rn(fmaf(__low2float(sg), d[0], __low2float(o)), fmaf(__high2float(sg), d[1], __high2float(o)));
    return *reinterpret_cast<const uint32_t*>(&g);
}

// Atoms whose gradient to add to is in flight: all of a warp's where the registers allow (binary16, 1080p, D = 72: 201 us with four and
// three blocks a multiprocessor, 160 with all nine and two; fp32: 317 with four and three blocks, 371 with nine and two; all with the slopes in registers).
template <typename CoefT, int AW> __host__ __device__ constexpr int ahead_of() { return Lane<CoefT>::PER == 2 && AW <= 9 ? AW : 4; }

template <typename CoefT, int AW, int WARPS, bool VEC, bool ADD>
__global__ void __launch_bounds__(WARPS * 32, resident_threads((AW + (ADD && VEC && ahead_of<CoefT, AW>() == AW ? AW : 0)) * NW) / (WARPS * 32))
balance_grad_kernel(const CoefT* __restrict__ coef, CoefT* __restrict__ grad, const __grid_constant__ BalanceGradParams p)
{
    using L = Lane<CoefT>;
    constexpr int PER = L::PER, PX = NW * PER, TP = 32 * PX;
    __shared__ __align__(16) float ssum[WARPS][TP];
    __shared__ __align__(16) float sdot[WARPS][TP];
    __shared__ float sa[AW * WARPS];                             // weighted slopes
    __shared__ __align__(16) float sk[TP];                       // 1 / S, 0 for a pixel that does not count
    __shared__ __align__(16) float sc[TP];                       // - mean weighted slope / S
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int f = blockIdx.x / p.tiles;
    const int64_t p0 = (int64_t)(blockIdx.x - f * p.tiles) * TP;
    const int D = p.D;
    const int64_t HW = p.HW;
    const int left = (int)min((int64_t)TP, HW - p0);
    const uint8_t* tile_mask = p.mask ? p.mask + (int64_t)f * HW + p0 : nullptr;
    uint32_t x[AW][NW], keep[NW];
    load_words<CoefT, AW, WARPS, VEC>(x, coef + (int64_t)f * D * HW + p0, HW, left, D, warp, lane);
    keep_words<CoefT, VEC>(keep, tile_mask, left, lane);
    // The weight goes into the slopes, not into 1 / S: weight / S is beyond fp32 for small S where the gradient, which has a slope's
    // size (about 1 / pixels) in it too, is not. In shared memory they leave the registers to the planes (1080p, D = 72, added: binary16
    // 160 -> 149 us, fp32 362 -> 299; written 100 -> 104, 192 both).
    if (tid < AW * WARPS) {
        const float weight = p.grad_loss ? p.weight * __ldg(p.grad_loss) : p.weight;
        sa[tid] = tid < D ? weight * __ldg(p.slope + (int64_t)f * D + tid) : 0.f;
    }
    __syncthreads();
    float sum[PX], dot[PX];
#pragma unroll
    for (int i = 0; i < PX; ++i) sum[i] = dot[i] = 0.f;
#pragma unroll
    for (int j = 0; j < AW; ++j) {
        const float a = sa[warp + j * WARPS];
        uint32_t m[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) m[w] = x[j][w] & keep[w];
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            const float v = L::get(m, i);
            sum[i] += v;
            dot[i] = fmaf(a, v, dot[i]);
        }
    }
    CoefT* dst = grad + ((int64_t)f * D + warp) * HW + p0 + (VEC ? lane * PX : lane);
    // what is added to is asked for ahead (a load cannot pass the stores before it)
    constexpr int AHEAD = ADD && VEC ? ahead_of<CoefT, AW>() : 1;
    uint4 ahead[AHEAD];
    auto ask = [&](int j) {
        if (warp + j * WARPS < D && lane * PX < left) ahead[j % AHEAD] = *reinterpret_cast<const uint4*>(dst + (int64_t)j * WARPS * HW);
    };
    if (ADD && VEC) {
#pragma unroll
        for (int j = 0; j < (AHEAD < AW ? AHEAD : AW); ++j) ask(j);
    }
    put_pixels<PX, VEC>(ssum[warp], sum, lane);
    put_pixels<PX, VEC>(sdot[warp], dot, lane);
    __syncthreads();
    if (tid < TP) {
        float S = 0.f, Q = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { S += ssum[w][tid]; Q += sdot[w][tid]; }
        const bool on = tid < left && !(S < kSmallestNormal) && (!tile_mask || __ldg(tile_mask + tid) != 0);
        const float r = 1.f / S;
        sk[tid] = on ? r : 0.f;
        sc[tid] = on ? -(Q * r) * r : 0.f;
    }
    __syncthreads();
    float k[PX], c[PX];
    get_pixels<PX, VEC>(k, sk, lane);
    get_pixels<PX, VEC>(c, sc, lane);
    bool all = true;                             // this warp's pixels all count
#pragma unroll
    for (int i = 0; i < PX; ++i) all &= k[i] != 0.f;
    all = __all_sync(0xffffffffu, all);
    auto finish = [&](auto every) {              // `every`: all pixels of the warp count
#pragma unroll
    for (int j = 0; j < AW; ++j) {
        if (warp + j * WARPS >= D) break;
        CoefT* to = dst + (int64_t)j * WARPS * HW;
        const float a = sa[warp + j * WARPS];
        uint32_t old[NW], o[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) old[w] = 0u;
        if (ADD) {
            if (VEC) {
                unpack(old, ahead[j % AHEAD]);
                if (j + AHEAD < AW) ask(j + AHEAD);
            } else {
#pragma unroll
                for (int i = 0; i < PX; ++i) L::put(old, i, lane + 32 * i < left ? L::one(to + 32 * i) : 0u);
            }
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            float d[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) d[i] = fmaf(a, k[w * PER + i], c[w * PER + i]);
            o[w] = result_word<ADD>((const CoefT*)nullptr, x[j][w], old[w], d);
            if (!decltype(every)::value) {       // a pixel that does not count keeps its bits, or is zero, whatever the weight is
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const uint32_t part = PER == 1 ? 0xFFFFFFFFu : 0xFFFFu << (16 * i);
                    if (k[w * PER + i] == 0.f) o[w] = (o[w] & ~part) | (old[w] & part);
                }
            }
        }
        if (VEC) {
            if (lane * PX < left) *reinterpret_cast<uint4*>(to) = make_uint4(o[0], o[1], o[2], o[3]);
        } else {
#pragma unroll
            for (int i = 0; i < PX; ++i) {
                if (lane + 32 * i < left) {
                    if (PER == 1) to[32 * i] = *reinterpret_cast<const CoefT*>(&o[i / PER]);
                    else reinterpret_cast<unsigned short*>(to)[32 * i] = (unsigned short)(i % 2 ? o[i / PER] >> 16 : o[i / PER] & 0xFFFFu);
                }
            }
        }
    }
    };
    if (all) finish(std::true_type{});
    else finish(std::false_type{});
}

// ---- host ------------------------------------------------------------------------------------------------------------------

int pixels_of_tile(int coef_dtype) { return coef_dtype == SR_F16 ? 256 : 128; }

// Blocks of a frame. Three blocks a multiprocessor over all frames, but no more than tiles.
int frame_blocks(int n, int64_t HW, int coef_dtype)
{
    const int64_t tiles = (HW + pixels_of_tile(coef_dtype) - 1) / pixels_of_tile(coef_dtype);
    int64_t want = (3ll * sm_count() + n - 1) / n;
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

// Atoms of a warp and warps of a block by D.
#define SR_BALANCE_BY_ATOMS(D, call)                                                                                                  \
    ((D) <= 16 ? call(2, 8) : (D) <= 32 ? call(4, 8) : (D) <= 48 ? call(6, 8) : (D) <= 72 ? call(9, 8) : (D) <= 96 ? call(12, 8) \
     : (D) <= 128 ? call(16, 8) : (D) <= 192 ? call(12, 16) : call(16, 16))

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
    if (cudaError_t e = launch_after(balance_sum_kernel, dim3(a.n, (a.D + kSumAtoms - 1) / kSumAtoms), kSumThreads, a.st, q)) return e;
    count_launches(2);
    return cudaSuccess;
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
