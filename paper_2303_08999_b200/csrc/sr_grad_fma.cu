// Gradients of the dictionary regression on the fp32 FMA pipe: every shape, fp32 or binary16 coefficients, all modes. The path of
// fp32 coefficients and the fallback for shapes the tensor-core kernels do not take.
//
//   G_j(i)          = sum_c grad_out_c(i) U_c(i + o_j)     per pixel, k*k values, never stored in global memory
//   grad_coef_l(i)  = sum_j dict[l][j] G_j(i)              grad_coef_kernel: one thread per pixel, G in registers
//   grad_dict[l][j] = sum_i coef_l(i) G_j(i)               grad_dict_kernel: a product [planes x pixels][pixels x k*k], a
//                                                          4 x 4 corner of it per thread, pixels staged in shared memory
// The first writes the coefficient-sized tensor and reads none, the second reads one and writes none, so two kernels move the
// bytes one would; what they do twice is G (c k^2 multiply-adds a pixel against D k^2).
#include "sr_train.cuh"

namespace sr {

namespace {

constexpr int TX = 32, CCHUNK = 4;

// The D k^2 multiply-adds of a pixel.
template <int K> struct KK { static constexpr int value = K * K, padded = (K * K + 3) & ~3; };

// Up-sampled tile of TX x TY pixels with its halo, CCHUNK channels at a time, in shared memory: the vertical taps on the LR columns that
// the tile reads, then the horizontal ones.
template <int K, int TY> struct UTile {
    static constexpr int P = (K - 1) / 2, UW = TX + 2 * P, UH = TY + 2 * P, LC = UW + 4;      // LR columns: most at scale 1
    float u[CCHUNK * UH * UW];
    float v[CCHUNK * UH * LC];
    int row0[UH], row_ph[UH], col0[UW], col_ph[UW];          // first tap of each row and column, and its phase
    float w[kMaxScale][4];

    __device__ __forceinline__ void taps(const Problem& pb, int X0, int Y0, int tid, int nthr)
    {
        for (int i = tid; i < UH + UW; i += nthr) {
            const bool row = i < UH;
            const int z = row ? clampi(Y0 - P + i, 0, pb.H - 1) : clampi(X0 - P + i - UH, 0, pb.W - 1);
            const int q = z / pb.r, ph = z - q * pb.r;
            if (row) { row0[i] = q + pb.ph.base[ph]; row_ph[i] = ph; }
            else { col0[i - UH] = q + pb.ph.base[ph]; col_ph[i - UH] = ph; }
        }
        for (int i = tid; i < kMaxScale * 4; i += nthr) w[i / 4][i % 4] = pb.ph.w[i / 4][i % 4];
    }
    // (between barriers of the threads; taps() before)
    __device__ __forceinline__ void fill(const float* __restrict__ lr, const Problem& pb, int f, int c0, int nc, int tid, int nthr)
    {
        const int lo = col0[0], nl = col0[UW - 1] + 4 - lo;
        for (int i = tid; i < nc * UH * LC; i += nthr) {
            const int line = i / LC, lc = i - line * LC;     // (constants)
            if (lc < nl) {
                const int ch = line / UH, uy = line - ch * UH;
                const float* col = lr + ((int64_t)f * pb.c + c0 + ch) * pb.h * pb.w + clampi(lo + lc, 0, pb.w - 1);
                const float* wy = w[row_ph[uy]];
                float acc = 0.f;
#pragma unroll
                for (int a = 0; a < 4; ++a) acc = fmaf(wy[a], __ldg(col + (int64_t)clampi(row0[uy] + a, 0, pb.h - 1) * pb.w), acc);
                v[i] = acc;
            }
        }
        __syncthreads();
        for (int i = tid; i < nc * UH * UW; i += nthr) {
            const int line = i / UW, ux = i - line * UW;
            const float* src = v + line * LC + col0[ux] - lo;
            const float* wx = w[col_ph[ux]];
            float acc = 0.f;
#pragma unroll
            for (int b = 0; b < 4; ++b) acc = fmaf(wx[b], src[b], acc);
            u[i] = acc;
        }
    }
};

__device__ __forceinline__ void store_coef(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store_coef(__half* p, int64_t i, float v) { p[i] = __float2half_rn(v); }

struct CoefGradParams {
    const float* lr;
    const uint8_t* idx;
    const float* gamma;
    const float* dict;
    const float* gout;
    int mode;
    int tiles_x, tiles_y, num_tiles;
    Problem pb;
};

template <int K, typename CoefT>
__global__ void __launch_bounds__(256)
grad_coef_kernel(const __grid_constant__ CoefGradParams p, CoefT* __restrict__ gcoef)
{
    constexpr int TY = 8, kk = KK<K>::value, kkp = KK<K>::padded, P = (K - 1) / 2;
    constexpr int UW = TX + 2 * P, UH = TY + 2 * P;
    extern __shared__ __align__(16) float smem[];
    __shared__ float sw[256];                    // global subset: the atom's weight
    __shared__ uint8_t satom[256];               // global subset: the atom of each plane
    __shared__ uint32_t slisted[8][256];         // lists: which atoms the pixel lists, a bit each
    const Problem& pb = p.pb;
    const int D = pb.D, s = pb.s, H = pb.H, W = pb.W;
    float* sdict = smem;                         // [D][kkp]
    UTile<K, TY>& ut = *reinterpret_cast<UTile<K, TY>*>(smem + (size_t)D * kkp);
    const int tid = threadIdx.y * TX + threadIdx.x;
    const int per = p.tiles_x * p.tiles_y;
    const int64_t HW = (int64_t)H * W;
    const bool compact = p.mode == kModeCompact || (p.mode == kModeGlobal && (pb.flags & SR_COEF_COMPACT));

    let_next_launch_start();                     // the dictionary's sums, which need nothing of this (128 x 128, fp32: 37 -> 29 us)
    for (int i = tid; i < D * kkp; i += 256) {
        const int l = i / kkp, j = i - l * kkp;
        sdict[i] = j < kk ? __ldg(p.dict + (int64_t)l * kk + j) : 0.f;
    }
    if (p.mode == kModeGlobal && tid == 0) {
        for (int l = 0; l < D; ++l) sw[l] = 0.f;
        for (int q = 0; q < s; ++q) {
            const int a = min((int)__ldg(p.idx + q), D - 1);
            const float g = p.gamma ? __ldg(p.gamma + q) : 1.f;
            satom[q] = (uint8_t)a;
            if (compact) sw[q] = g;
            else sw[a] += g;                     // an atom listed twice counts with both weights
        }
    }
  for (int t = blockIdx.x; t < p.num_tiles; t += gridDim.x) {
    const int f = t / per, rest = t - f * per;
    const int ty = rest / p.tiles_x, tx = rest - ty * p.tiles_x;
    const int X0 = tx * TX, Y0 = ty * TY, X = X0 + threadIdx.x, Y = Y0 + threadIdx.y;
    const bool valid = X < W && Y < H;
    const int64_t pix = (int64_t)min(Y, H - 1) * W + min(X, W - 1);
    float G[kkp];
#pragma unroll
    for (int j = 0; j < kkp; ++j) G[j] = 0.f;
    __syncthreads();
    ut.taps(pb, X0, Y0, tid, 256);
    for (int c0 = 0; c0 < pb.c; c0 += CCHUNK) {
        const int nc = min(CCHUNK, pb.c - c0);
        __syncthreads();
        ut.fill(p.lr, pb, f, c0, nc, tid, 256);
        __syncthreads();
        for (int ch = 0; ch < nc; ++ch) {
            const float g = valid ? __ldg(p.gout + ((int64_t)f * pb.c + c0 + ch) * HW + pix) : 0.f;
            const float* u = ut.u + ch * UH * UW + threadIdx.y * UW + threadIdx.x;
#pragma unroll
            for (int a = 0; a < K; ++a)
#pragma unroll
                for (int b = 0; b < K; ++b) G[a * K + b] = fmaf(g, u[a * UW + b], G[a * K + b]);
        }
    }
    auto dot = [&](int atom) {
        const float4* row = reinterpret_cast<const float4*>(sdict + atom * kkp);
        float acc[4] = {0.f, 0.f, 0.f, 0.f};     // four chains
#pragma unroll
        for (int j4 = 0; j4 < kkp / 4; ++j4) {
            const float4 dv = row[j4];
            acc[0] = fmaf(dv.x, G[4 * j4 + 0], acc[0]);
            acc[1] = fmaf(dv.y, G[4 * j4 + 1], acc[1]);
            acc[2] = fmaf(dv.z, G[4 * j4 + 2], acc[2]);
            acc[3] = fmaf(dv.w, G[4 * j4 + 3], acc[3]);
        }
        return (acc[0] + acc[1]) + (acc[2] + acc[3]);
    };
    const int planes = compact ? s : D;
    CoefT* out = gcoef + (int64_t)f * planes * HW + pix;
    if (p.mode == kModeCompact) {
        const uint8_t* list = p.idx + (int64_t)f * s * HW + pix;
        for (int q0 = 0; q0 < s; q0 += 8) {      // (eight loads in flight)
            int a[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = q0 + i < s ? min((int)__ldg(list + (int64_t)(q0 + i) * HW), D - 1) : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (q0 + i < s) {
                    const float v = dot(a[i]);
                    if (valid) store_coef(out, (int64_t)(q0 + i) * HW, v);
                }
        }
    } else if (p.mode == kModeGlobal) {
        for (int q = 0; q < planes; ++q) {
            const float w = sw[q];
            const float v = w != 0.f ? w * dot(compact ? satom[q] : q) : 0.f;
            if (valid) store_coef(out, (int64_t)q * HW, v);
        }
    } else if (p.mode == kModeIdx) {
        for (int i = 0; i < (D + 31) / 32; ++i) slisted[i][tid] = 0u;
        for (int q = 0; q < s; ++q) {
            const int a = min((int)__ldg(p.idx + ((int64_t)f * s + q) * HW + pix), D - 1);
            slisted[a >> 5][tid] |= 1u << (a & 31);
        }
        for (int l = 0; l < D; ++l) {
            const float v = dot(l);
            if (valid) store_coef(out, (int64_t)l * HW, (slisted[l >> 5][tid] >> (l & 31)) & 1u ? v : 0.f);
        }
    } else {
        for (int l = 0; l < D; ++l) {
            const float v = dot(l);
            if (valid) store_coef(out, (int64_t)l * HW, v);
        }
    }
  }
}

struct DictGradParams {
    const float* lr;
    const uint8_t* idx;
    const float* gout;
    float* partial;              // [slot][rows][kk]
    int mode;
    int rows;                    // planes whose sums are wanted (D, or s of a subset)
    int chunk;                   // planes a block works on (gridDim.y chunks)
    int ahead;                   // planes arrive by asynchronous copies of this many bytes (16 or 4), a tile ahead; 0 = not
    int tiles_x, tiles_y, num_tiles;
    Problem pb;
};

// A block owns a chunk of planes and walks tiles of 32 x 4 pixels. Per tile: G of every pixel and the planes' coefficients in
// shared memory, pixels innermost; then thread (row group, tap group, share of the pixels) adds its 4 x 4 corner. The corner of a
// tile is summed by itself and then added to the running one, so that a long frame adds few numbers of like size.
template <int K, typename CoefT>
__global__ void __launch_bounds__(256)
grad_dict_kernel(const __grid_constant__ DictGradParams p, const CoefT* __restrict__ coef)
{
    constexpr int TY = 4, NPX = TX * TY, kk = KK<K>::value, kkp = KK<K>::padded, P = (K - 1) / 2;
    constexpr int UW = TX + 2 * P, UH = TY + 2 * P;
    constexpr int PITCH = NPX + 4;               // rows four banks apart: 16-byte reads of eight rows touch every bank once
    constexpr int TG = kkp / 4;                  // tap groups
    extern __shared__ __align__(16) float smem[];
    const Problem& pb = p.pb;
    const int D = pb.D, s = pb.s, H = pb.H, W = pb.W, tid = threadIdx.x;
    const int64_t HW = (int64_t)H * W;
    const int row0 = blockIdx.y * p.chunk, nrow = min(p.chunk, p.rows - row0);
    const int rgroups = (nrow + 3) / 4, items = rgroups * TG;
    float* sG = smem;                            // [kkp][PITCH]
    float* sPhi = sG + kkp * PITCH;              // [chunk rounded up to 4][PITCH]
    const int phi = ((p.chunk + 3) & ~3) * PITCH;        // floats of a buffer of planes (two where they arrive by asynchronous copies)
    UTile<K, TY>& ut = *reinterpret_cast<UTile<K, TY>*>(sPhi + (size_t)phi * (p.ahead ? 2 : 1));
    const int shares = max(1, 256 / items);      // threads that split the pixels of one corner
    const int share = tid / items, item = tid - share * items;
    const int rg = item / TG, tg = item - rg * TG;
    const bool works = share < shares;

    for (int i = tid; i < kkp * PITCH; i += 256) sG[i] = 0.f;
    for (int i = tid; i < phi * (p.ahead ? 2 : 1); i += 256) sPhi[i] = 0.f;
    // A tile's planes by asynchronous copies of `ahead` bytes, a tile ahead (fp32, whole planes): 1080p x4, D = 72: 1584 -> 743 us.
    auto fetch = [&](int t, float* to) {
        const int per = p.tiles_x * p.tiles_y;
        const int f = t / per, rest = t - f * per;
        const int ty = rest / p.tiles_x, X0 = (rest - ty * p.tiles_x) * TX, Y0 = ty * TY;
        const bool compact = (pb.flags & SR_COEF_COMPACT) != 0;
        const int units = p.ahead == 16 ? NPX / 4 : NPX, step = p.ahead / 4;
        for (int i = tid; i < nrow * units; i += 256) {
            const int q = i / units, px = (i - q * units) * step, X = X0 + px % TX, Y = Y0 + px / TX;        // (units: 32 or 128)
            int64_t plane;
            if (p.mode == kModeGlobal) plane = compact ? (int64_t)f * s + row0 + q : (int64_t)f * D + min((int)__ldg(p.idx + row0 + q), D - 1);
            else plane = (int64_t)f * D + row0 + q;
            const bool in = X < W && Y < H;                              // (W a multiple of four where a copy is four pixels)
            const CoefT* src = coef + plane * HW + (in ? (int64_t)Y * W + X : 0);
            const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to + q * PITCH + px);
            if (step == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int buf = 0;
    if (p.ahead) {
        __syncthreads();
        if ((int)blockIdx.x < p.num_tiles) fetch(blockIdx.x, sPhi);
    }
    float total[4][4] = {};
    for (int t = blockIdx.x; t < p.num_tiles; t += gridDim.x) {
        const int per = p.tiles_x * p.tiles_y;
        const int f = t / per, rest = t - f * per;
        const int ty = rest / p.tiles_x, tx = rest - ty * p.tiles_x;
        const int X0 = tx * TX, Y0 = ty * TY;
        // ---- the planes' coefficients (zero outside the image)
        __syncthreads();
        const float* planes = sPhi + (p.ahead ? buf * phi : 0);
        if (p.ahead) {
            if (t + (int)gridDim.x < p.num_tiles) fetch(t + gridDim.x, sPhi + (buf ^ 1) * phi);
            buf ^= 1;
        } else if (p.mode == kModeIdx || p.mode == kModeCompact) {
            for (int i = tid; i < nrow * NPX; i += 256) sPhi[(i / NPX) * PITCH + i % NPX] = 0.f;
            __syncthreads();
            for (int i = tid; i < s * NPX; i += 256) {
                const int q = i / NPX, px = i - q * NPX, X = X0 + px % TX, Y = Y0 + px / TX;
                if (X < W && Y < H) {
                    const int64_t pix = (int64_t)Y * W + X;
                    const int a = min((int)__ldg(p.idx + ((int64_t)f * s + q) * HW + pix), D - 1);
                    if (a >= row0 && a < row0 + nrow)
                        sPhi[(a - row0) * PITCH + px] = load_coef(coef, (p.mode == kModeCompact ? (int64_t)f * s + q : (int64_t)f * D + a) * HW + pix);
                }
            }
        } else {
            const bool compact = (pb.flags & SR_COEF_COMPACT) != 0;
            for (int i = tid; i < nrow * NPX; i += 256) {
                const int q = i / NPX, px = i - q * NPX, X = X0 + px % TX, Y = Y0 + px / TX;
                int64_t plane;
                if (p.mode == kModeGlobal) plane = compact ? (int64_t)f * s + row0 + q : (int64_t)f * D + min((int)__ldg(p.idx + row0 + q), D - 1);
                else plane = (int64_t)f * D + row0 + q;
                sPhi[q * PITCH + px] = X < W && Y < H ? load_coef(coef, plane * HW + (int64_t)Y * W + X) : 0.f;
            }
        }
        // ---- G: two threads a pixel, every other patch row each
        const int px = tid % NPX, half = tid / NPX;
        const int gx = X0 + px % TX, gy = Y0 + px / TX;
        const bool valid = gx < W && gy < H;
        ut.taps(pb, X0, Y0, tid, 256);
        for (int c0 = 0; c0 < pb.c; c0 += CCHUNK) {
            const int nc = min(CCHUNK, pb.c - c0);
            __syncthreads();
            ut.fill(p.lr, pb, f, c0, nc, tid, 256);
            __syncthreads();
            float g[CCHUNK];
#pragma unroll
            for (int ch = 0; ch < CCHUNK; ++ch)
                g[ch] = valid && ch < nc ? __ldg(p.gout + ((int64_t)f * pb.c + c0 + ch) * HW + (int64_t)gy * W + gx) : 0.f;
            for (int a = half; a < K; a += 2) {
#pragma unroll
                for (int b = 0; b < K; ++b) {
                    float v = c0 == 0 ? 0.f : sG[(a * K + b) * PITCH + px];
#pragma unroll
                    for (int ch = 0; ch < CCHUNK; ++ch)
                        if (ch < nc) v = fmaf(g[ch], ut.u[(ch * UH + px / TX + a) * UW + px % TX + b], v);
                    sG[(a * K + b) * PITCH + px] = valid ? v : 0.f;
                }
            }
        }
        if (p.ahead) {                           // this tile's planes have landed; the next one's may travel on
            if (t + (int)gridDim.x < p.num_tiles) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        // ---- the corner
        if (works) {
            float acc[4][4] = {};
            for (int q = share; q < NPX / 4; q += shares) {
                float4 a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(planes + (4 * rg + i) * PITCH + 4 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = *reinterpret_cast<const float4*>(sG + (4 * tg + i) * PITCH + 4 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = fmaf(a[i].w, b[j].w, fmaf(a[i].z, b[j].z, fmaf(a[i].y, b[j].y, fmaf(a[i].x, b[j].x, acc[i][j]))));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) total[i][j] += acc[i][j];
        }
    }
    // ---- the shares of a corner, one after the other (fixed order), then to the block's slot
    __syncthreads();
    float* sum = smem;                           // [items][16]
    for (int sh = 0; sh < shares; ++sh) {
        if (share == sh) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[item * 16 + i] = (sh ? sum[item * 16 + i] : 0.f) + total[i / 4][i % 4];
        }
        __syncthreads();
    }
    if (share == 0) {
        float* out = p.partial + (int64_t)blockIdx.x * p.rows * kk;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 4 * rg + i / 4, j = 4 * tg + i % 4;
            if (r < nrow && j < kk) out[(int64_t)(row0 + r) * kk + j] = sum[item * 16 + i];
        }
    }
    wait_for_launch_before();                    // (the coefficients' kernel beside it: whoever waits for this launch waits for both)
}

// Sums the slots. A block takes 32 neighbouring elements of one plane row's flat range, eight threads to an element, and adds
// the eight in a fixed order; fp64, because the partial sums are as large as the whole.
__global__ void __launch_bounds__(256)
grad_dict_sum_kernel(const float* __restrict__ partial, int slots, int elems, float* __restrict__ gdict)
{
    __shared__ double part[8][33];
    const int e = blockIdx.x * 32 + threadIdx.x % 32, g = threadIdx.x / 32;
    wait_for_launch_before();
    double acc = 0.0;
    if (e < elems) {
#pragma unroll 8
        for (int i = g; i < slots; i += 8) acc += (double)__ldg(partial + (int64_t)i * elems + e);
    }
    part[g][threadIdx.x % 32] = acc;
    __syncthreads();
    if (g == 0 && e < elems) {
        for (int i = 1; i < 8; ++i) acc += part[i][threadIdx.x];
        gdict[e] = (float)acc;
    }
}

// The same for a subset: block q sums the taps of plane q, writes the re-weight's gradient sum_j dict[a_q][j] A_q[j], and, if it
// is the first plane of its atom, the atom's row sum of gamma A over the planes of that atom. Blocks s .. s + D - 1 write the
// zero rows of the atoms outside the subset.
__global__ void __launch_bounds__(256)
grad_subset_sum_kernel(const float* __restrict__ partial, int slots, int s, int D, int kk, const uint8_t* __restrict__ idx,
                       const float* __restrict__ gamma, const float* __restrict__ dict, float* __restrict__ gdict, float* __restrict__ ggamma)
{
    __shared__ double part[8][81];
    __shared__ double rowsum[81];
    const int tid = threadIdx.x;
    wait_for_launch_before();
    if ((int)blockIdx.x >= s) {
        const int l = blockIdx.x - s;
        bool in = false;
        for (int q = 0; q < s; ++q) in |= min((int)__ldg(idx + q), D - 1) == l;
        if (!in && gdict)
            for (int j = tid; j < kk; j += 256) gdict[(int64_t)l * kk + j] = 0.f;
        return;
    }
    const int q = blockIdx.x, atom = min((int)__ldg(idx + q), D - 1);
    bool first = true;
    for (int i = 0; i < q; ++i) first &= min((int)__ldg(idx + i), D - 1) != atom;
    for (int j = tid; j < kk; j += 256) rowsum[j] = 0.0;
    for (int q2 = q; q2 < s; ++q2) {
        if (q2 != q && (!first || !gdict || min((int)__ldg(idx + q2), D - 1) != atom)) continue;
        __syncthreads();
        for (int i = tid; i < 8 * kk; i += 256) {
            const int g = i / kk, j = i - g * kk;
            double acc = 0.0;
#pragma unroll 8
            for (int sl = g; sl < slots; sl += 8) acc += (double)__ldg(partial + ((int64_t)sl * s + q2) * kk + j);
            part[g][j] = acc;
        }
        __syncthreads();
        if (tid < kk) {
            double acc = 0.0;
            for (int g = 0; g < 8; ++g) acc += part[g][tid];
            part[0][tid] = acc;
            rowsum[tid] += (gamma ? (double)__ldg(gamma + q2) : 1.0) * acc;
        }
        __syncthreads();
        if (q2 == q && ggamma && tid == 0) {
            double acc = 0.0;
            for (int j = 0; j < kk; ++j) acc += (double)__ldg(dict + (int64_t)atom * kk + j) * part[0][j];
            ggamma[q] = (float)acc;
        }
    }
    __syncthreads();
    if (first && gdict && tid < kk) gdict[(int64_t)atom * kk + tid] = (float)rowsum[tid];
}

template <int K, typename CoefT> cudaError_t launch_coef_t(const GradArgs& a)
{
    constexpr int TY = 8;
    const Problem& pb = a.pb;
    CoefGradParams p{a.lr, a.idx, a.gamma, a.dict, a.gout, a.mode, (pb.W + TX - 1) / TX, (pb.H + TY - 1) / TY, 0, pb};
    const int64_t tiles = (int64_t)p.tiles_x * p.tiles_y * pb.n;
    if (tiles > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    p.num_tiles = (int)tiles;
    const int blocks = (int)(tiles < 4 * sm_count() ? tiles : 4 * sm_count());
    const size_t smem = (size_t)pb.D * KK<K>::padded * sizeof(float) + sizeof(UTile<K, TY>);
    auto kern = grad_coef_kernel<K, CoefT>;
    constexpr size_t most = 256 * KK<K>::padded * sizeof(float) + sizeof(UTile<K, TY>);        // 256 atoms
    static bool done[64] = {false};
    if (cudaError_t e = allow_most_smem(kern, most, done)) return e;
    kern<<<blocks, dim3(TX, TY), smem, a.st>>>(p, static_cast<CoefT*>(a.gcoef));
    count_launches(1);
    return cudaGetLastError();
}

template <int K, typename CoefT> cudaError_t launch_dict_t(const GradArgs& a, int* slots)
{
    constexpr int TY = 4, TG = KK<K>::padded / 4, PITCH = TX * TY + 4;
    const Problem& pb = a.pb;
    DictGradParams p{};
    p.lr = a.lr; p.idx = a.idx; p.gout = a.gout; p.partial = a.scratch; p.mode = a.mode; p.pb = pb;
    p.rows = grad_rows(a);
    // planes of a block: at most 256 corners of 4 x 4, and 80 planes (shared memory)
    constexpr int kMost = 4 * (256 / TG) < 80 ? 4 * (256 / TG) : 80;
    const int chunks = (p.rows + kMost - 1) / kMost;
    p.chunk = ((p.rows + chunks - 1) / chunks + 3) & ~3;
    p.tiles_x = (pb.W + TX - 1) / TX;
    p.tiles_y = (pb.H + TY - 1) / TY;
    const int64_t tiles = (int64_t)p.tiles_x * p.tiles_y * pb.n;
    if (tiles > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    p.num_tiles = (int)tiles;
    const int gx = (int)(tiles < grad_slots() ? tiles : grad_slots());
    const bool whole = a.mode == kModeDense || a.mode == kModeGlobal;
    p.ahead = sizeof(CoefT) == 4 && whole ? (pb.W % 4 == 0 && ((uintptr_t)a.coef & 15) == 0 ? 16 : 4) : 0;
    size_t smem = ((size_t)KK<K>::padded + (size_t)p.chunk * (p.ahead ? 2 : 1)) * PITCH * sizeof(float) + sizeof(UTile<K, TY>);
    const size_t sums = (size_t)((p.chunk + 3) / 4) * TG * 16 * sizeof(float);
    if (smem < sums) smem = sums;
    auto kern = grad_dict_kernel<K, CoefT>;
    constexpr size_t planes = (kMost + 3) & ~3, most_sums = planes / 4 * TG * 16 * sizeof(float);
    constexpr size_t most_tiles = (KK<K>::padded + planes * 2) * PITCH * sizeof(float) + sizeof(UTile<K, TY>), most = most_tiles > most_sums ? most_tiles : most_sums;
    static bool done[64] = {false};
    if (cudaError_t e = allow_most_smem(kern, most, done)) return e;
    count_launches(1);
    *slots = gx;
    // Early only behind this call's own coefficient kernel, which started after everything before the call; behind another kernel this one
    // would read inputs that are still being written, if that one lets the next launch start.
    return launch_after_smem(kern, dim3(gx, (p.rows + p.chunk - 1) / p.chunk), 256, smem, a.st, a.gcoef != nullptr, p, static_cast<const CoefT*>(a.coef));
}

template <typename CoefT> cudaError_t launch_coef_k(const GradArgs& a)
{
    switch (a.pb.k) {
    case 1: return launch_coef_t<1, CoefT>(a);
    case 3: return launch_coef_t<3, CoefT>(a);
    case 5: return launch_coef_t<5, CoefT>(a);
    case 7: return launch_coef_t<7, CoefT>(a);
    default: return launch_coef_t<9, CoefT>(a);
    }
}

template <typename CoefT> cudaError_t launch_dict_k(const GradArgs& a, int* slots)
{
    switch (a.pb.k) {
    case 1: return launch_dict_t<1, CoefT>(a, slots);
    case 3: return launch_dict_t<3, CoefT>(a, slots);
    case 5: return launch_dict_t<5, CoefT>(a, slots);
    case 7: return launch_dict_t<7, CoefT>(a, slots);
    default: return launch_dict_t<9, CoefT>(a, slots);
    }
}

} // namespace

cudaError_t launch_grad_coef_fma(const GradArgs& a)
{
    return a.coef_dtype == SR_F16 ? launch_coef_k<__half>(a) : launch_coef_k<float>(a);
}

cudaError_t launch_grad_dict_fma(const GradArgs& a, int* slots)
{
    return a.coef_dtype == SR_F16 ? launch_dict_k<__half>(a, slots) : launch_dict_k<float>(a, slots);
}

cudaError_t launch_grad_dict_sum(const GradArgs& a, int slots)
{
    const int kk = a.pb.k * a.pb.k;
    const float* partial = a.scratch;
    count_launches(1);
    if (a.mode == kModeGlobal)
        return launch_after(grad_subset_sum_kernel, dim3(a.pb.s + a.pb.D), 256, a.st, partial, slots, a.pb.s, a.pb.D, kk, a.idx, a.gamma, a.dict, a.gdict, a.ggamma);
    const int elems = a.pb.D * kk;
    return launch_after(grad_dict_sum_kernel, dim3((elems + 31) / 32), 256, a.st, partial, slots, elems, a.gdict);
}

} // namespace sr
