// Balance loss of a per-pixel selection and its gradient.
//   share p_l(i) = |coef_l(i)| / S(i), S(i) = sum_m |coef_m(i)|;  f_l = counts_l / (s T);  loss = D sum_l f_l mean_i p_l(i)
//   dL/dcoef_l(i) = sign(coef_l) / S(i) (a_l - sum_m a_m p_m(i)),  a_l = D f_l / T (the slope)
//
// Both directions stream the [n][D][H][W] planes once and are bound by that. A block takes a tile of 256 (binary16) or 128 (fp32)
// pixels with all its atoms: warp w holds atoms w, w + WARPS, ... of the tile in registers, as loaded (a lane: 16 bytes of each), and adds
// their magnitudes; the warps' sums meet in shared memory, where one thread a pixel finishes them; then every warp works on from its
// registers, so the planes are read from memory once although a share needs the whole column first. Widening costs an instruction
// an element, so magnitudes and signs are taken on the packed words.
#include "sr_train.cuh"

namespace sr {

namespace {

constexpr float kSmallestNormal = 1.17549435e-38f;

// A lane's share of one atom of a tile: four 32-bit words, PX pixels. VEC: neighbouring pixels, one 16-byte access (planes and bases
// that allow it); else the words' elements are 32 pixels apart, so that single-element accesses of a warp are one run.
template <typename CoefT> struct Lane;
template <> struct Lane<float> {
    static constexpr int PX = 4;
    static constexpr uint32_t kMagnitude = 0x7FFFFFFFu;
    static __device__ __forceinline__ float get(const uint32_t (&v)[4], int i) { return __uint_as_float(v[i]); }
    static __device__ __forceinline__ uint32_t one(const float* p) { return __float_as_uint(__ldcs(p)); }
    static __device__ __forceinline__ void put(uint32_t (&v)[4], int i, uint32_t x) { v[i] = x; }
    static __device__ __forceinline__ uint32_t keep(const bool (&on)[4], int j) { return on[j] ? kMagnitude : 0u; }
};
template <> struct Lane<__half> {
    static constexpr int PX = 8;
    static constexpr uint32_t kMagnitude = 0x7FFF7FFFu;
    static __device__ __forceinline__ float get(const uint32_t (&v)[4], int i)
    {
        const __half2 h = *reinterpret_cast<const __half2*>(&v[i / 2]);
        return i % 2 ? __high2float(h) : __low2float(h);
    }
    static __device__ __forceinline__ uint32_t one(const __half* p) { return (uint32_t)__half_as_ushort(__ldcs(p)); }
    static __device__ __forceinline__ void put(uint32_t (&v)[4], int i, uint32_t x) { v[i / 2] = i % 2 ? __byte_perm(v[i / 2], x, 0x5410) : x; }
    static __device__ __forceinline__ uint32_t keep(const bool (&on)[8], int j) { return (on[2 * j] ? 0x7FFFu : 0u) | (on[2 * j + 1] ? 0x7FFF0000u : 0u); }
};

template <int PX, bool VEC> __device__ __forceinline__ int slot_pixel(int lane, int i) { return VEC ? lane * PX + i : lane + 32 * i; }

// The tile's words of this warp's atoms; zero beyond the frame's end.
template <typename CoefT, int AW, int WARPS, bool VEC>
__device__ __forceinline__ void load_words(uint32_t (&x)[AW][4], const CoefT* tile, int64_t HW, int left, int D, int warp, int lane)
{
    using L = Lane<CoefT>;
    const CoefT* src = tile + (int64_t)warp * HW + (VEC ? lane * L::PX : lane);
    const bool whole = left >= 32 * L::PX;
#pragma unroll
    for (int a = 0; a < AW; ++a, src += WARPS * HW) {
        x[a][0] = x[a][1] = x[a][2] = x[a][3] = 0u;
        if (warp + a * WARPS < D) {
            if (VEC) {
                if (lane * L::PX < left) {
                    const uint4 t = __ldcs(reinterpret_cast<const uint4*>(src));
                    x[a][0] = t.x; x[a][1] = t.y; x[a][2] = t.z; x[a][3] = t.w;
                }
            } else if (whole) {
#pragma unroll
                for (int i = 0; i < L::PX; ++i) L::put(x[a], i, L::one(src + 32 * i));
            } else {
#pragma unroll
                for (int i = 0; i < L::PX; ++i) L::put(x[a], i, lane + 32 * i < left ? L::one(src + 32 * i) : 0u);
            }
        }
    }
}

// What to keep of each word: its magnitude bits, nothing of pixels that do not count (whatever stands there).
template <typename CoefT, bool VEC>
__device__ __forceinline__ void keep_words(uint32_t (&keep)[4], const uint8_t* mask, int left, int lane)
{
    using L = Lane<CoefT>;
#pragma unroll
    for (int j = 0; j < 4; ++j) keep[j] = L::kMagnitude;
    if (mask) {
        bool on[L::PX];
#pragma unroll
        for (int i = 0; i < L::PX; ++i) {
            const int px = slot_pixel<L::PX, VEC>(lane, i);
            on[i] = px < left && __ldg(mask + px) != 0;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) keep[j] = L::keep(on, j);
    }
}

template <int PX, bool VEC> __device__ __forceinline__ void put_pixels(float* row, const float (&v)[PX], int lane)
{
    if (VEC) {
#pragma unroll
        for (int j = 0; j < PX / 4; ++j) *reinterpret_cast<float4*>(row + lane * PX + 4 * j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < PX; ++i) row[lane + 32 * i] = v[i];
    }
}
template <int PX, bool VEC> __device__ __forceinline__ void get_pixels(float (&v)[PX], const float* row, int lane)
{
    if (VEC) {
#pragma unroll
        for (int j = 0; j < PX / 4; ++j) {
            const float4 t = *reinterpret_cast<const float4*>(row + lane * PX + 4 * j);
            v[4 * j] = t.x; v[4 * j + 1] = t.y; v[4 * j + 2] = t.z; v[4 * j + 3] = t.w;
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

// (blocks a multiprocessor: as many as the registers of AW atoms allow)
template <typename CoefT, int AW, int WARPS, bool VEC>
__global__ void __launch_bounds__(WARPS * 32, (AW <= 9 ? 768 : 512) / (WARPS * 32))
balance_kernel(const CoefT* __restrict__ coef, const __grid_constant__ BalanceParams p)
{
    using L = Lane<CoefT>;
    constexpr int PX = L::PX, TP = 32 * PX, NT = WARPS * 32, RANKS = NT / TP;   // threads a pixel
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
        uint32_t x[AW][4], keep[4];
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
            for (int j = 0; j < 4; ++j) x[a][j] &= keep[j];
#pragma unroll
            for (int i = 0; i < PX; ++i) sum[i] += L::get(x[a], i);
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

// Block (atoms 8 a .. 8 a + 7, frame f) adds up the frame's partial sums, 128 threads to an atom and a tree of fixed shape; the block
// that finishes last then knows every frame's sums and writes slopes and loss.
constexpr int kSumAtoms = 8;
__global__ void __launch_bounds__(1024)
balance_sum_kernel(const __grid_constant__ BalanceSumParams p)
{
    __shared__ double ssum[1024];
    __shared__ int scnt[1024];
    __shared__ int svalid;
    __shared__ bool last;
    const int tid = threadIdx.x, f = blockIdx.x, D = p.D, i8 = tid % kSumAtoms, g = tid / kSumAtoms, l = blockIdx.y * kSumAtoms + i8;
    if (tid == 0) svalid = 0;
    wait_for_launch_before();
    __syncthreads();
    double acc = 0.0;
    int c = 0, v = 0;
#pragma unroll 4
    for (int b = g; b < p.bx; b += 1024 / kSumAtoms) {
        const int64_t row = (int64_t)f * p.bx + b;
        if (l < D) {
            acc += (double)__ldg(p.part_share + row * D + l);
            c += __ldg(p.part_count + row * (D + 1) + l);
        }
        if (i8 == 0) v += __ldg(p.part_count + row * (D + 1) + D);
    }
    v = __reduce_add_sync(0xffffffffu, v);
    if (tid % 32 == 0) atomicAdd(&svalid, v);
    ssum[tid] = acc;
    scnt[tid] = c;
    for (int o = 512; o >= kSumAtoms; o >>= 1) {
        __syncthreads();
        if (tid < o) { ssum[tid] += ssum[tid + o]; scnt[tid] += scnt[tid + o]; }
    }
    __syncthreads();
    const int valid = svalid;
    if (tid < kSumAtoms && l < D) {
        p.share_sum[(int64_t)f * D + l] = ssum[tid];
        p.counts[(int64_t)f * D + l] = scnt[tid];
        p.share[(int64_t)f * D + l] = valid ? (float)(ssum[tid] / valid) : 0.f;
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

// Two results of a word: the factor of the magnitude with the coefficient's sign, zero where the coefficient is.
template <bool ADD> __device__ __forceinline__ uint32_t result_word(const float*, uint32_t x, uint32_t old, const float* d)
{
    const float g = __uint_as_float(x) == 0.f ? 0.f : __uint_as_float(__float_as_uint(d[0]) ^ (x & 0x80000000u));
    return __float_as_uint(ADD ? __uint_as_float(old) + g : g);
}
template <bool ADD> __device__ __forceinline__ uint32_t result_word(const __half*, uint32_t x, uint32_t old, const float* d)
{
    const __half2 h = *reinterpret_cast<const __half2*>(&x);
    const uint32_t some = __hne2_mask(h, __half2half2(__ushort_as_half(0)));       // (NaN != 0)
    if (!ADD) {                                  // rounding is symmetric: the sign may come after it
        const __half2 g = __floats2half2_rn(d[0], d[1]);
        return (*reinterpret_cast<const uint32_t*>(&g) ^ (x & 0x80008000u)) & some;
    }
    const float g0 = (some & 1u) ? __uint_as_float(__float_as_uint(d[0]) ^ ((x & 0x8000u) << 16)) : 0.f;
    const float g1 = (some >> 31) ? __uint_as_float(__float_as_uint(d[1]) ^ (x & 0x80000000u)) : 0.f;
    const __half2 o = *reinterpret_cast<const __half2*>(&old);
    const __half2 g = __floats2half2_rn(__low2float(o) + g0, __high2float(o) + g1);
    return *reinterpret_cast<const uint32_t*>(&g);
}

template <typename CoefT, int AW, int WARPS, bool VEC, bool ADD>
__global__ void __launch_bounds__(WARPS * 32, (AW <= 9 ? 768 : 512) / (WARPS * 32))
balance_grad_kernel(const CoefT* __restrict__ coef, CoefT* __restrict__ grad, const __grid_constant__ BalanceGradParams p)
{
    using L = Lane<CoefT>;
    constexpr int PX = L::PX, TP = 32 * PX, PER = PX / 4;        // elements of a word
    __shared__ __align__(16) float ssum[WARPS][TP];
    __shared__ __align__(16) float sdot[WARPS][TP];
    __shared__ __align__(16) float sk[TP];                       // weight / S
    __shared__ __align__(16) float sc[TP];                       // - mean slope * weight / S
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int f = blockIdx.x / p.tiles;
    const int64_t p0 = (int64_t)(blockIdx.x - f * p.tiles) * TP;
    const int D = p.D;
    const int64_t HW = p.HW;
    const int left = (int)min((int64_t)TP, HW - p0);
    const uint8_t* tile_mask = p.mask ? p.mask + (int64_t)f * HW + p0 : nullptr;
    uint32_t x[AW][4], keep[4];
    load_words<CoefT, AW, WARPS, VEC>(x, coef + (int64_t)f * D * HW + p0, HW, left, D, warp, lane);
    keep_words<CoefT, VEC>(keep, tile_mask, left, lane);
    float a[AW];
#pragma unroll
    for (int j = 0; j < AW; ++j) a[j] = warp + j * WARPS < D ? __ldg(p.slope + (int64_t)f * D + warp + j * WARPS) : 0.f;
    float sum[PX], dot[PX];
#pragma unroll
    for (int i = 0; i < PX; ++i) sum[i] = dot[i] = 0.f;
#pragma unroll
    for (int j = 0; j < AW; ++j) {
        uint32_t m[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) m[w] = x[j][w] & keep[w];
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            const float v = L::get(m, i);
            sum[i] += v;
            dot[i] = fmaf(a[j], v, dot[i]);
        }
    }
    put_pixels<PX, VEC>(ssum[warp], sum, lane);
    put_pixels<PX, VEC>(sdot[warp], dot, lane);
    __syncthreads();
    if (tid < TP) {
        float S = 0.f, Q = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { S += ssum[w][tid]; Q += sdot[w][tid]; }
        const float weight = p.grad_loss ? p.weight * __ldg(p.grad_loss) : p.weight;
        const bool on = tid < left && !(S < kSmallestNormal) && (!tile_mask || __ldg(tile_mask + tid) != 0);
        const float r = 1.f / S, k = on ? weight * r : 0.f;
        sk[tid] = k;
        sc[tid] = on ? -(Q * r) * k : 0.f;
    }
    __syncthreads();
    float k[PX], c[PX];
    get_pixels<PX, VEC>(k, sk, lane);
    get_pixels<PX, VEC>(c, sc, lane);
    CoefT* dst = grad + ((int64_t)f * D + warp) * HW + p0 + (VEC ? lane * PX : lane);
#pragma unroll
    for (int j = 0; j < AW; ++j, dst += WARPS * HW) {
        if (warp + j * WARPS >= D) break;
        uint32_t old[4] = {0u, 0u, 0u, 0u}, o[4];
        if (ADD) {
            if (VEC) {
                if (lane * PX < left) {
                    const uint4 t = *reinterpret_cast<const uint4*>(dst);
                    old[0] = t.x; old[1] = t.y; old[2] = t.z; old[3] = t.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < PX; ++i) L::put(old, i, lane + 32 * i < left ? L::one(dst + 32 * i) : 0u);
            }
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            float d[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) d[i] = fmaf(a[j], k[w * PER + i], c[w * PER + i]);
            o[w] = result_word<ADD>((const CoefT*)nullptr, x[j][w], old[w], d);
            if (ADD) {                           // a pixel that does not count keeps its bits
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const uint32_t part = PER == 1 ? 0xFFFFFFFFu : 0xFFFFu << (16 * i);
                    if (k[w * PER + i] == 0.f) o[w] = (o[w] & ~part) | (old[w] & part);
                }
            }
        }
        if (VEC) {
            if (lane * PX < left) *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
        } else {
#pragma unroll
            for (int i = 0; i < PX; ++i) {
                if (lane + 32 * i < left) {
                    if (PER == 1) dst[32 * i] = *reinterpret_cast<const CoefT*>(&o[i / PER]);
                    else reinterpret_cast<unsigned short*>(dst)[32 * i] = (unsigned short)(i % 2 ? o[i / PER] >> 16 : o[i / PER] & 0xFFFFu);
                }
            }
        }
    }
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

// Atoms of a warp (registers) and warps of a block by D.
#define SR_BALANCE_BY_ATOMS(D, call)                                   \
    ((D) <= 16 ? call(2, 8) : (D) <= 32 ? call(4, 8) : (D) <= 48 ? call(6, 8) : (D) <= 72 ? call(9, 8) : (D) <= 80 ? call(10, 8) : (D) <= 128 ? call(8, 16) : call(16, 16))

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
    if (cudaError_t e = launch_after(balance_sum_kernel, dim3(a.n, (a.D + kSumAtoms - 1) / kSumAtoms), 1024, a.st, q)) return e;
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
