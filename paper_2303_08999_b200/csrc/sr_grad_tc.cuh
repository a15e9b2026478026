// What the tensor-core kernels of the regression's gradients share (sr_grad_tc.cu, sr_grad_roles.cu): the layout of G and of the atoms, the
// up-sampled tile, and the host's set-up.
#pragma once

#include "sr_ptx.cuh"
#include "sr_tile_upsample.cuh"
#include "sr_train.cuh"

namespace sr {
namespace gradtc {

using namespace ptx;
using namespace tile;

constexpr int kGroupThreads = 128;             // a group: a row of 128 pixels, one a thread
constexpr int kOutBytes = 16384;                // 128 atoms by 64 pixels on their way to global memory
constexpr int kMaxTH = 8, kMaxC = 4;

template <int K> struct GGeo {
    static constexpr int kk = K * K, P = (K - 1) / 2, UW = tile_uw(P);
    static constexpr int BLOCKS = kk > 32 ? 2 : 1;                 // 128-byte columns of a G row: hi | lo side by side, or one each
    static constexpr int LO_CHUNK = kk > 32 ? 0 : 4;               // 16-byte unit where lo starts inside its column
    static constexpr int KSTEPS = (kk + 15) / 16;                  // K-steps of the first product
    static constexpr int CHUNKS = 2 * KSTEPS;                      // 16-byte units that are written
    static constexpr int G_BYTES = BLOCKS * 128 * 128;
    static constexpr int NB = kk > 32 ? 128 : 64;                  // N of the second product: hi and lo columns
    static constexpr int LO_COL = kk > 32 ? 64 : 32;
};

struct GradTcParams {
    Geom g;
    const float* lr;
    const float* dict;
    const float* gout;
    const uint8_t* idx;
    const float* gamma;
    const __half* coef;
    __half* gcoef;
    float* partial;
    int* status;
    int mode;
    int rows;                    // planes of the product: D, or s of a compact subset (first product); D, or s of a subset (second)
    int planes;                  // planes of a frame in coef / gcoef
    int stage_bytes, chunk_bytes;
    int own_out;                 // first product: bytes of a group's buffer for results; 0 = they pass through the G tile
    int tma;                     // second product: coefficients arrive by TMA
    long long wait_cycles;
    int lose;                    // test hook: the first commit of block 0 is left out
};

struct __align__(16) GradCtl {
    uint64_t mma[2];             // a row's product is complete (of the two groups of sr_grad_tc.cu)
    uint64_t full[2];            // a row's coefficients have landed
    uint64_t drain;
    WaitCtx wait;
    uint32_t tmem_base;
    unsigned top_g[2], top_l[2]; // largest finite |grad_out| and |lr| of a tile, as bits; by tile parity
    float wpad[kMaxScale][12];
    uint8_t atoms[256];          // atom of each plane (subset)
};

__device__ __forceinline__ bool group_barrier_and(int id, bool pred)
{
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 128, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((int)pred), "r"(id) : "memory");
    return r != 0;
}
// TMA store of a box (innermost coordinate a multiple of eight elements); wait until such stores have read their source, or are done.
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, const void* src, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"((uint64_t)map), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// mbar_wait for waits of some hundred cycles: polls without suspending the thread. Bounded like it.
__device__ __forceinline__ bool mbar_wait_short(uint64_t* bar, uint32_t parity, volatile WaitCtx* wc)
{
    const uint32_t at = smem_u32(bar);
    const long long t0 = clock64();
    while (true) {
#pragma unroll 1
        for (int i = 0; i < 32; ++i) {
            uint32_t done;
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(done) : "r"(at), "r"(parity) : "memory");
            if (done) return true;
        }
        if (wc->abort_flag) return false;
        if (clock64() - t0 > const_cast<const WaitCtx*>(wc)->limit) {
            wc->abort_flag = 1;
            return false;
        }
    }
}
// One lane of a converged warp, known to the compiler as such (operands of what it issues stay in uniform registers).
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void cp_async_wait_all_() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ unsigned finite_bits(float v) { const unsigned b = __float_as_uint(v) & 0x7FFFFFFFu; return b < 0x7F800000u ? b : 0u; }
__device__ __forceinline__ int exponent_of(unsigned bits) { return bits ? max((int)(bits >> 23), 1) - 127 : -127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }   // -126 .. 127

// hi + lo of two values, packed.
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo)
{
    const __half2 h = __floats2half2_rn(a, b);
    const __half2 l = __floats2half2_rn(a - __low2float(h), b - __high2float(h));
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
}

// Writes the kk values v of row `row` as hi + lo into a [rows][128 B] tile (swizzled); block_bytes: distance of the two columns.
template <int K> __device__ __forceinline__ void write_row(uint8_t* tile, int block_bytes, int row, const float (&v)[K * K])
{
    using G = GGeo<K>;
    uint8_t* base = tile + row * 128;
    const int x = row & 7;
#pragma unroll
    for (int c = 0; c < G::CHUNKS; ++c) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = 8 * c + 2 * i;
            const float a = j < G::kk ? v[j < G::kk ? j : 0] : 0.f, b = j + 1 < G::kk ? v[j + 1 < G::kk ? j + 1 : 0] : 0.f;
            split2(a, b, h[i], l[i]);
        }
        *reinterpret_cast<uint4*>(base + ((c ^ x) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(base + (G::BLOCKS - 1) * block_bytes + (((c + G::LO_CHUNK) ^ x) << 4)) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// Shared memory of the kernels: [operand tiles, 1024-byte aligned][sU][sV][sL][sg].
struct Floats { float *U, *V, *L, *g; };
__device__ __forceinline__ Floats carve_floats(uint8_t* at, const GradTcParams& p, int UW)
{
    Floats f;
    f.U = reinterpret_cast<float*>(at);
    f.V = f.U + p.g.pb.c * p.g.uh * UW;
    f.L = f.V + p.g.pb.c * p.g.uh * p.g.tcols;
    f.g = f.L + p.g.pb.c * p.g.trows * p.g.tcols + 8;            // (the horizontal pass reads a few values beyond its own)
    return f;
}

// ---- what the kernels do per tile --------------------------------------------------------------------------------------------

// Barrier of the threads that make a tile: the block, or its first NT threads.
template <int NT, bool NAMED> __device__ __forceinline__ bool makers_and(bool ok)
{
    if (!NAMED) return __syncthreads_and(ok) != 0;
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, %2, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((int)ok), "n"(NT) : "memory");
    return r != 0;
}
template <int NT, bool NAMED> __device__ __forceinline__ void makers_sync()
{
    if (!NAMED) __syncthreads();
    else asm volatile("barrier.cta.sync 1, %0;" ::"n"(NT) : "memory");
}

// The tiles of a block: blockIdx.x, blockIdx.x + gridDim.x, ..., without a division a tile. (Blocks at work stay in one band of rows: runs
// of tiles down the strips instead, 1080p x4, subset of eight: 222 us against 169.)
struct Tiles {
    int t, n, base;                              // tile, its number among the block's, the number of its first row
    int tx, ty, f, sx, sy, sf;                   // position and step as (column, row, frame)
    int x0, y0, rows;
    __device__ __forceinline__ explicit Tiles(const Geom& g) : t(blockIdx.x), n(0), base(0)
    {
        const int step = gridDim.x, per = g.tiles_x * g.tiles_y;
        f = t / per; ty = (t - f * per) / g.tiles_x; tx = t - f * per - ty * g.tiles_x;
        sf = step / per; sy = (step - sf * per) / g.tiles_x; sx = step - sf * per - sy * g.tiles_x;
        place(g);
    }
    __device__ __forceinline__ void place(const Geom& g) { x0 = tx * TW; y0 = ty * g.th; rows = min(g.th, g.pb.H - y0); }
    __device__ __forceinline__ bool more(const Geom& g) const { return t < g.num_tiles; }
    __device__ __forceinline__ void next(const Geom& g)
    {
        base += rows;
        ++n;
        t += gridDim.x;
        tx += sx; if (tx >= g.tiles_x) { tx -= g.tiles_x; ++ty; }
        ty += sy; if (ty >= g.tiles_y) { ty -= g.tiles_y; ++f; }
        f += sf;
        place(g);
    }
};

// The up-sampled tile, the pixel's grad_out values of the group's rows and the tile's scale; made by NG groups.
template <int K, int NG, bool NAMED> struct TileState {
    using G = GGeo<K>;
    static constexpr int NT = NG * kGroupThreads, ROWS = (kMaxTH + NG - 1) / NG;
    LrWindow w;                                  // of the tile in work
    float next_g[ROWS][kMaxC];                   // grad_out of the next tile's rows, asked for a tile ahead
    float scale, unscale;

    // rows first, first + NG, ... of the pixel's column
    __device__ __forceinline__ void ask_g(const GradTcParams& p, const LrWindow& t, int first, int x)
    {
        const Problem& pb = p.g.pb;
        const int64_t HW = (int64_t)pb.H * pb.W;
        const float* src = p.gout + (int64_t)t.f * pb.c * HW + (int64_t)(t.y0 + first) * pb.W + t.x0 + x;
        const bool inside = t.x0 + x < pb.W;
#pragma unroll
        for (int i = 0; i < ROWS; ++i, src += NG * pb.W) {
            const bool on = inside && first + NG * i < t.rows;
            const float* at = src;
#pragma unroll
            for (int c = 0; c < kMaxC; ++c, at += HW)
                if (c < pb.c) next_g[i][c] = on ? __ldg(at) : 0.f;       // (pb.c is uniform)
        }
    }

    __device__ __forceinline__ void take(const GradTcParams& p, const Tiles& tl, const Floats& s, int tid, int first)
    {
        w.f = tl.f; w.y0 = tl.y0; w.x0 = tl.x0; w.rows = tl.rows;
        lr_window_of_tile<G::P>(p.g, w);
        prefetch_lr_window_of(p.g, p.lr, w, s.L, tid, NT);
        ask_g(p, w, first, tid % kGroupThreads);
    }

    __device__ __forceinline__ void start(const GradTcParams& p, const Tiles& tl, const Floats& s, int tid, int first)
    {
        if (tl.more(p.g)) take(p, tl, s, tid, first);
    }

    // All NT threads. `ok` comes back the same for all of them; the tile may be read when it is true. first, next_first: the group's first
    // row of this tile and of the next one. unscale_out: where one thread leaves the factor that takes results back.
    __device__ __forceinline__ bool make(const GradTcParams& p, GradCtl& ctl, const Tiles& after, int parity, const Floats& s, int tid, bool ok, int first,
                                         int next_first, float* unscale_out)
    {
        const int C = p.g.pb.c, uh = w.rows + 2 * G::P, x = tid % kGroupThreads;
        cp_async_wait_all_();
        ok = makers_and<NT, NAMED>(ok);          // LR window landed, the previous tile left by every thread
        if (!ok) return false;
        const int nv = p.g.tcols / 4, v_lanes = NT / nv;
        if (tid / nv < v_lanes) vertical_pass(p.g, w, uh, G::P, s.L, s.V, 4 * (tid % nv), tid / nv, v_lanes);
        unsigned top = 0;
        for (int i = tid; i < C * w.nrows * nv; i += NT) {
            const int row = fast_div(i, nv, p.g.tc4_magic), c4 = i - row * nv;
            if (c4 < w.nc4) {
                const float4 v = *reinterpret_cast<const float4*>(s.L + row * p.g.tcols + 4 * c4);
                top = max(top, max(max(finite_bits(v.x), finite_bits(v.y)), max(finite_bits(v.z), finite_bits(v.w))));
            }
        }
        unsigned top_g = 0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int c = 0; c < kMaxC; ++c) {
                if (c < C && (kMaxTH % NG == 0 || first + NG * i < kMaxTH)) {
                    s.g[((first + NG * i) * C + c) * kGroupThreads + x] = next_g[i][c];
                    top_g = max(top_g, finite_bits(next_g[i][c]));
                }
            }
        top = __reduce_max_sync(0xffffffffu, top);
        top_g = __reduce_max_sync(0xffffffffu, top_g);
        if ((tid & 31) == 0) { atomicMax(&ctl.top_l[parity], top); atomicMax(&ctl.top_g[parity], top_g); }
        makers_sync<NT, NAMED>();
        const LrWindow now = w;
        if (after.more(p.g)) take(p, after, s, tid, next_first);
        if (tid == 0) { ctl.top_l[parity ^ 1] = 0; ctl.top_g[parity ^ 1] = 0; }
        // |G| <= c max|g| 1.375^2 max|lr| < 2^(eg + el + 5) for up to four channels: scaled below 2^15
        const int eg = exponent_of(ctl.top_g[parity]), el = max(exponent_of(ctl.top_l[parity]), -100);
        const int a = min(max(10 - eg - el, -126), 126);
        scale = power_of_two(a);
        unscale = power_of_two(-a);
        if (tid == 0 && unscale_out) *unscale_out = unscale;
        const int nh = G::UW / 4, h_lanes = NT / nh;
        if (tid / nh < h_lanes) horizontal_pass<G::P>(p.g, ctl.wpad, now, uh, s.V, s.U, tid % nh, tid / nh, h_lanes);
        makers_sync<NT, NAMED>();
        return true;
    }
};

// G of a pixel, times the tile's scale. `between` is called after the first channel. One and three channels are written out: a loop
// over channels carries its k*k sums from register to register (293 instructions a row and warp for three, 5 x 5).
template <int K, int NC, typename Between>
__device__ __forceinline__ void patch_grad_c(const float* u, int u_channel, const float* g, int C, float scale, float (&G)[K * K], Between between)
{
    constexpr int UW = GGeo<K>::UW;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c < C) {
            const float gv = g[c * kGroupThreads] * scale;
#pragma unroll
            for (int a = 0; a < K; ++a)
#pragma unroll
                for (int b = 0; b < K; ++b) {
                    const float v = u[c * u_channel + a * UW + b];
                    G[a * K + b] = c == 0 ? gv * v : fmaf(gv, v, G[a * K + b]);
                }
        }
        if (c == 0) between();
    }
}
template <int K, typename Between>
__device__ __forceinline__ void patch_grad(const float* u, int u_channel, const float* g, int C, float scale, float (&G)[K * K], Between between)
{
    if (C == 3) patch_grad_c<K, 3>(u, u_channel, g, 3, scale, G, between);
    else if (C == 1) patch_grad_c<K, 1>(u, u_channel, g, 1, scale, G, between);
    else patch_grad_c<K, kMaxC>(u, u_channel, g, C, scale, G, between);
}

__device__ __forceinline__ void init_ctl(GradCtl& ctl, const GradTcParams& p, int tid, int nthr, int drains)
{
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) { mbar_init(&ctl.mma[i], 1); mbar_init(&ctl.full[i], 1); }
        mbar_init(&ctl.drain, drains);
        ctl.wait.abort_flag = 0;
        ctl.wait.limit = p.wait_cycles;
        ctl.top_g[0] = ctl.top_g[1] = ctl.top_l[0] = ctl.top_l[1] = 0;
        fence_barrier_init();
    }
    fill_wpad(p.g.pb, ctl.wpad, tid, nthr);
}

// Plane q's atom as a row of the first product's operand: its taps, times the plane's weight where a subset has one, times a power of two
// that brings the largest to [2^9, 2^10). Returns what takes results back, 0 for a plane outside the subset.
template <int K> __device__ __forceinline__ float write_atom(const GradTcParams& p, uint8_t* sD, int d_block, int q)
{
    using G = GGeo<K>;
    const Problem& pb = p.g.pb;
    const int D = pb.D;
    int atom = q;
    float weight = 1.f;
    if (p.mode == kModeGlobal) {
        weight = 0.f;
        if (pb.flags & SR_COEF_COMPACT) {
            atom = min((int)__ldg(p.idx + q), D - 1);
            weight = p.gamma ? __ldg(p.gamma + q) : 1.f;
        } else {
            for (int i = 0; i < pb.s; ++i)
                if (min((int)__ldg(p.idx + i), D - 1) == q) weight += p.gamma ? __ldg(p.gamma + i) : 1.f;
        }
    }
    float v[G::kk];
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < G::kk; ++j) { v[j] = weight * __ldg(p.dict + (int64_t)atom * G::kk + j); top = max(top, finite_bits(v[j])); }
    const int e = min(max(9 - exponent_of(top), -126), 126);
    const float up = power_of_two(e);
#pragma unroll
    for (int j = 0; j < G::kk; ++j) v[j] *= up;
    write_row<K>(sD, d_block, q, v);
    return weight != 0.f ? power_of_two(-e) : 0.f;
}

// ---- host ------------------------------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
        return (EncodeTiledFn)f;
    }();
    return fn;
}

inline int smem_optin()
{
    static int cache[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (!cache[dev]) {
        int v = 0, major = 0;
        if (cudaDeviceGetAttribute(&v, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess) return 0;
        if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return 0;
        cache[dev] = major == 10 ? v : -1;
    }
    return cache[dev];
}

constexpr int kStaticReserve = 4096;

// Tile height: eight rows, fewer on frames that eight would leave multiprocessors without a tile.
inline int tile_rows(const Problem& pb)
{
    const int64_t columns = (int64_t)((pb.W + TW - 1) / TW) * pb.n;
    for (int th = kMaxTH; th > 2; th /= 2)
        if (columns * ((pb.H + th - 1) / th) >= 2 * sm_count()) return th;
    return 2;
}

template <int K> size_t float_bytes(Geom& g, const Problem& pb, const float* lr)
{
    return (plan_geom(g, pb, tile_rows(pb), lr) + 8 + (size_t)kMaxTH * pb.c * kGroupThreads) * sizeof(float);
}

template <typename Kern> cudaError_t allow_smem(Kern kern, bool (&done)[64], int reserve = kStaticReserve)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!done[dev]) {
        if (cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin() - reserve)) return e;
        done[dev] = true;
    }
    return cudaSuccess;
}

// A [n][planes][H][W] binary16 tensor in boxes of 64 pixels of one row by `box_planes` planes, 128-byte swizzle.
inline bool encode_planes(CUtensorMap* map, const void* base, const Problem& pb, int planes, int box_planes)
{
    const cuuint64_t dims[4] = {(cuuint64_t)pb.W, (cuuint64_t)pb.H, (cuuint64_t)planes, (cuuint64_t)pb.n};
    const cuuint64_t strides[3] = {(cuuint64_t)pb.W * 2, (cuuint64_t)pb.W * pb.H * 2, (cuuint64_t)pb.W * pb.H * 2 * planes};
    const cuuint32_t es[4] = {1, 1, 1, 1}, box[4] = {64, 1, (cuuint32_t)box_planes, 1};
    return encode_fn() && encode_fn()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
                                      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline int stage_bytes_of(int rows) { return 2 * ((rows + 7) & ~7) * 128; }

inline GradTcParams common_params(const GradArgs& a)
{
    GradTcParams p{};
    p.lr = a.lr; p.dict = a.dict; p.gout = a.gout; p.idx = a.idx; p.gamma = a.gamma;
    p.coef = static_cast<const __half*>(a.coef);
    p.gcoef = static_cast<__half*>(a.gcoef);
    p.partial = a.scratch;
    p.status = device_status_word();
    p.mode = a.mode;
    p.planes = (a.mode == kModeCompact || (a.mode == kModeGlobal && (a.pb.flags & SR_COEF_COMPACT))) ? a.pb.s : a.pb.D;
    p.wait_cycles = wait_cycle_limit();
    p.lose = take_injected_lost_arrival() ? 1 : 0;
    return p;
}

inline bool form_supported(const GradArgs& a)
{
    const Problem& pb = a.pb;
    return a.coef_dtype == SR_F16 && (pb.k == 3 || pb.k == 5 || pb.k == 7) && pb.c <= kMaxC && smem_optin() > 0 &&
           (int64_t)((pb.W + TW - 1) / TW) * ((pb.H + 1) / 2) * pb.n <= 0x7FFFFFFF;
}

inline bool fits(size_t smem, int reserve = kStaticReserve) { return smem + reserve <= (size_t)smem_optin(); }

} // namespace gradtc
} // namespace sr
