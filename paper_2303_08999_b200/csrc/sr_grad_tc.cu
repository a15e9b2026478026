// Gradients of the dictionary regression on the tcgen05 tensor cores, for binary16 coefficients: k in {3, 5, 7}, up to four channels,
// any width and number of atoms.
//
//   grad_coef: per row of 128 pixels, a product [pixels x k*k][k*k x atoms]       (grad_coef_tc_kernel)
//   grad_dict: per row of 128 pixels, a product [atoms x pixels][pixels x k*k]    (grad_dict_tc_kernel), summed over rows
//
// Both share their operand G_j(i) = sum_c grad_out_c(i) U_c(i + o_j), computed by one thread per pixel from the up-sampled tile in
// shared memory and written as two binary16 numbers hi + lo (22 bits) into a [128 pixels][128 bytes] tile under the 128-byte
// swizzle. Read along its rows it is the K-major operand of the first product, read across them the MN-major operand of
// the second. Binary16 has few exponents, so G is scaled by a power of two per tile (from the largest finite grad_out and LR
// value the tile can meet) and each atom by one of its own; the results are scaled back in fp32.
//
// A thread block is two groups of four warps; a group takes every other row of the block's tile and runs on its own barriers, so
// that with two blocks on a multiprocessor four rows are in different stages of  G -> tensor core -> results  at any time.
// Every wait is bounded, as in the forward kernels.
#include "sr_ptx.cuh"
#include "sr_tile_upsample.cuh"
#include "sr_train.cuh"

namespace sr {

namespace {

using namespace ptx;
using namespace tile;

constexpr int kThreads = 256, kGroups = 2, kGroupThreads = 128;
constexpr int kOutBytes = 16384;                // 128 atoms by 64 pixels on their way to global memory
constexpr int kMaxTH = 8, kMaxRowsOfGroup = kMaxTH / kGroups, kMaxC = 4;

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
    uint64_t mma[kGroups];       // a row's product is complete
    uint64_t full[kGroups];      // a row's coefficients have landed
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
// Waits of a row's length (some hundred cycles): tested without the time hint of mbar_wait, whose sleep is longer than they are
// (1080p x4, D = 72, k = 5: coefficients 137 -> 104 us, dictionary 129 -> 98). Bounded like it.
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

// ---- what both kernels do per tile -----------------------------------------------------------------------------------------

// The up-sampled tile, the pixel's grad_out values of the group's rows and the tile's scale.
template <int K> struct TileState {
    using G = GGeo<K>;
    LrWindow w;                                  // of the tile in work
    float next_g[kMaxRowsOfGroup][kMaxC];        // grad_out of the next tile's rows, asked for a tile ahead
    float scale, unscale;

    __device__ __forceinline__ void ask_g(const GradTcParams& p, const LrWindow& t, int grp, int x)
    {
        const int64_t HW = (int64_t)p.g.pb.H * p.g.pb.W;
#pragma unroll
        for (int i = 0; i < kMaxRowsOfGroup; ++i) {
            const int row = grp + kGroups * i;
            const float* src = p.gout + (int64_t)t.f * p.g.pb.c * HW + (int64_t)(t.y0 + row) * p.g.pb.W + t.x0 + x;
#pragma unroll
            for (int c = 0; c < kMaxC; ++c) next_g[i][c] = row < t.rows && c < p.g.pb.c && t.x0 + x < p.g.pb.W ? __ldg(src + c * HW) : 0.f;
        }
    }

    __device__ __forceinline__ void start(const GradTcParams& p, float* sL, int tid)
    {
        if ((int)blockIdx.x < p.g.num_tiles) {
            lr_window<G::P>(p.g, blockIdx.x, w);
            prefetch_lr_window_of(p.g, p.lr, w, sL, tid, kThreads);
            ask_g(p, w, tid / kGroupThreads, tid % kGroupThreads);
        }
    }

    // All threads. `ok` comes back the same for the whole block; the tile may be read when it is true.
    __device__ __forceinline__ bool make(const GradTcParams& p, GradCtl& ctl, int t, int parity, float* sL, float* sV, float* sU, float* sg, int tid, bool ok)
    {
        const int C = p.g.pb.c, uh = w.rows + 2 * G::P, grp = tid / kGroupThreads, x = tid % kGroupThreads;
        cp_async_wait_all_();
        ok = __syncthreads_and(ok) != 0;         // LR window landed, the previous tile left by every thread
        if (!ok) return false;
        const int nv = p.g.tcols / 4, v_lanes = kThreads / nv;
        if (tid / nv < v_lanes) vertical_pass(p.g, w, uh, G::P, sL, sV, 4 * (tid % nv), tid / nv, v_lanes);
        unsigned top = 0;
        for (int i = tid; i < C * w.nrows * nv; i += kThreads) {
            const int row = fast_div(i, nv, p.g.tc4_magic), c4 = i - row * nv;
            if (c4 < w.nc4) {
                const float4 v = *reinterpret_cast<const float4*>(sL + row * p.g.tcols + 4 * c4);
                top = max(top, max(max(finite_bits(v.x), finite_bits(v.y)), max(finite_bits(v.z), finite_bits(v.w))));
            }
        }
        unsigned top_g = 0;
#pragma unroll
        for (int i = 0; i < kMaxRowsOfGroup; ++i)
#pragma unroll
            for (int c = 0; c < kMaxC; ++c) {
                if (c < C) {
                    sg[((grp + kGroups * i) * C + c) * kGroupThreads + x] = next_g[i][c];
                    top_g = max(top_g, finite_bits(next_g[i][c]));
                }
            }
        top = __reduce_max_sync(0xffffffffu, top);
        top_g = __reduce_max_sync(0xffffffffu, top_g);
        if ((tid & 31) == 0) { atomicMax(&ctl.top_l[parity], top); atomicMax(&ctl.top_g[parity], top_g); }
        __syncthreads();
        const LrWindow now = w;
        if (t + (int)gridDim.x < p.g.num_tiles) {
            lr_window<G::P>(p.g, t + gridDim.x, w);
            prefetch_lr_window_of(p.g, p.lr, w, sL, tid, kThreads);
            ask_g(p, w, grp, x);
        }
        if (tid == 0) { ctl.top_l[parity ^ 1] = 0; ctl.top_g[parity ^ 1] = 0; }
        const int nh = G::UW / 4, h_lanes = kThreads / nh;
        if (tid / nh < h_lanes) horizontal_pass<G::P>(p.g, ctl.wpad, now, uh, sV, sU, tid % nh, tid / nh, h_lanes);
        __syncthreads();
        // |G| <= c max|g| 1.375^2 max|lr| < 2^(eg + el + 5) for up to four channels: scaled below 2^15
        const int eg = exponent_of(ctl.top_g[parity]), el = max(exponent_of(ctl.top_l[parity]), -100);
        const int a = min(max(10 - eg - el, -126), 126);
        scale = power_of_two(a);
        unscale = power_of_two(-a);
        return true;
    }
};

// G of a pixel, times the tile's scale. `between` is called after the first channel. One and three channels are written out: a loop
// over channels carries its k*k sums from register to register (293 instructions a row and warp for three, 5 x 5; 165 written out).
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

__device__ __forceinline__ void init_ctl(GradCtl& ctl, const GradTcParams& p, int tid)
{
    if (tid == 0) {
        for (int i = 0; i < kGroups; ++i) { mbar_init(&ctl.mma[i], 1); mbar_init(&ctl.full[i], 1); }
        mbar_init(&ctl.drain, kGroups);
        ctl.wait.abort_flag = 0;
        ctl.wait.limit = p.wait_cycles;
        ctl.top_g[0] = ctl.top_g[1] = ctl.top_l[0] = ctl.top_l[1] = 0;
        fence_barrier_init();
    }
    fill_wpad(p.g.pb, ctl.wpad, tid, kThreads);
}

// Shared memory of both kernels: [operand tiles, 1024-byte aligned][sU][sV][sL][sg].
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

// ---- gradient of the coefficients ------------------------------------------------------------------------------------------

// The first product in one of two layouts of its result.
//   ATOMS: accumulator lane = atom, column = pixel (atoms are the rows of the product). A warp puts its 32 atoms' values of 64 pixels
//          into 4 KB of shared memory (a buffer of its own, or its part of the G tile, which the product has read by then) and one TMA store takes them to
//          their planes; needs W % 8 == 0. Storing a lane's row directly, 32 bytes at a time, touches 32 planes an instruction: 268 us
//          at 1080p x4, D = 72, where one value of one plane per instruction (below) takes 223.
//   else:  lane = pixel, column = atom. A thread stores its pixel's value of one plane after the other, 64 bytes a warp, whatever the
//          alignment.
template <int K, bool ATOMS>
__global__ void __launch_bounds__(kThreads, 2)
grad_coef_tc_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ GradTcParams p)
{
    using G = GGeo<K>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ GradCtl ctl;
    __shared__ float sback[256];                 // 2^e of each plane's atom (0: a plane outside the subset)
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const Problem& pb = p.g.pb;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), grp = warp / (kGroupThreads / 32), x = tid % kGroupThreads, lane = tid & 31;
    const bool leads = warp % (kGroupThreads / 32) == 0;         // the group's first warp: its elected lane issues what one thread issues
    const int C = pb.c, D = pb.D, W = pb.W, rows_pad = (p.rows + 15) & ~15;
    uint8_t* sG = smem + grp * G::G_BYTES;
    uint8_t* sD = smem + kGroups * G::G_BYTES;   // [column][rows_pad][128 B]
    const int d_block = rows_pad * 128;
    // results on their way out: behind the atoms (4 KB for each warp that has some), or in the G tile
    uint8_t* sOut = ATOMS && p.own_out ? sD + G::BLOCKS * d_block + grp * p.own_out : sG;
    const Floats s = carve_floats(sD + G::BLOCKS * d_block + (ATOMS ? kGroups * p.own_out : 0), p, G::UW);

    init_ctl(ctl, p, tid);
    for (int i = tid; i < (kGroups * G::G_BYTES + G::BLOCKS * d_block) / 16; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    for (int i = tid; i < p.g.pb.c * p.g.trows * p.g.tcols + 8; i += kThreads) s.L[i] = 0.f;
    __syncthreads();
    TileState<K> ts;
    ts.start(p, s.L, tid);
    // the atoms, each times a power of two that brings its largest tap to [2^9, 2^10)
    for (int q = tid; q < p.rows; q += kThreads) {
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
        sback[q] = weight != 0.f ? power_of_two(-e) : 0.f;
    }
    fence_proxy_async_smem();
    if (warp == 0) tmem_alloc(&ctl.tmem_base, kGroups * 128);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = ctl.tmem_base + grp * 128;
    volatile WaitCtx* wc = &ctl.wait;
    const int64_t HW = (int64_t)pb.H * W;
    const uint64_t g_desc = make_smem_desc(smem_u32(sG), 16, 1024, kSwizzle128B);
    const uint64_t d_desc = make_smem_desc(smem_u32(sD), 16, 1024, kSwizzle128B);
    constexpr uint32_t kGLo = (G::BLOCKS == 2 ? 128 * 128 : G::LO_CHUNK * 16) >> 4;
    const uint32_t kDLo = (uint32_t)(G::BLOCKS == 2 ? d_block : G::LO_CHUNK * 16) >> 4;
    bool lose = p.lose != 0 && blockIdx.x == 0 && warp == 0;
    uint32_t phase = 0;
    bool ok = true;
    int parity = 0;
    for (int t = blockIdx.x; t < p.g.num_tiles; t += gridDim.x, parity ^= 1) {
        const LrWindow w = ts.w;
        if (!(ok = ts.make(p, ctl, t, parity, s.L, s.V, s.U, s.g, tid, ok))) break;
        const bool inside = w.x0 + x < W;
        const uint32_t at = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        auto multiply = [&](int m0) {            // thread 0 of the group: planes m0 .. m0 + 127 of the row in sG
            tc_fence_after_sync();
            const int nr = min(128, p.rows - m0);
            const uint32_t idesc = make_idesc_f16(128, ATOMS ? 128 : (nr + 15) & ~15, false, false);
            const uint64_t dd = d_desc + (uint64_t)((uint32_t)m0 * 128u >> 4);
#pragma unroll
            for (int ks = 0; ks < G::KSTEPS; ++ks) {
                const uint64_t gh = g_desc + 2 * ks, gl = gh + kGLo, dh = dd + 2 * ks, dl = dh + kDLo;
                mma_f16_ss(tmem, ATOMS ? dh : gh, ATOMS ? gh : dh, idesc, ks > 0);
                mma_f16_ss(tmem, ATOMS ? dh : gl, ATOMS ? gl : dh, idesc, 1u);
                mma_f16_ss(tmem, ATOMS ? dl : gh, ATOMS ? gh : dl, idesc, 1u);
            }
            if (!lose) mma_commit(&ctl.mma[grp]);
            lose = false;
        };
        // The results of a row whose product has been started. False: the group leaves (all of it).
        auto finish = [&](int row) {
            const int64_t pix = (int64_t)(w.y0 + row) * W + w.x0 + x;
            for (int m0 = 0; m0 < p.rows; m0 += 128) {
                const int nr = min(128, p.rows - m0);
                if (m0 > 0) {
                    tc_fence_before_sync();
                    if (!group_barrier_and(1 + grp, ok)) return false;
                    if (leads && elect_one()) multiply(m0);
                    __syncwarp();
                }
                ok = __all_sync(0xffffffffu, ok && mbar_wait_short(&ctl.mma[grp], phase, wc));
                phase ^= 1;
                tc_fence_after_sync();
                if (!ok) continue;               // (the next barrier tells the group)
                if (ATOMS) {
                    const int l = 32 * (warp & 3) + lane;
                    if (l - lane < nr) {
                        const float back = l < nr ? sback[m0 + l] : 0.f, k = back * ts.unscale;
                        uint8_t* mine = sOut + (warp & 3) * (kOutBytes / 4);
#pragma unroll
                        for (int c0 = 0; c0 < 128; c0 += 64) {
                            uint32_t h[32];
#pragma unroll
                            for (int c1 = 0; c1 < 64; c1 += 32) {
                                float acc[32];
                                tmem_ld_x16(at + c0 + c1, acc);
                                tmem_ld_x16(at + c0 + c1 + 16, acc + 16);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const __half2 v2 = __floats2half2_rn(acc[2 * i] * k, acc[2 * i + 1] * k);
                                    h[c1 / 2 + i] = *reinterpret_cast<const uint32_t*>(&v2);
                                }
                            }
                            if (back == 0.f) {               // outside the subset: zeros, whatever G is
#pragma unroll
                                for (int i = 0; i < 32; ++i) h[i] = 0u;
                            }
                            if (lane == 0) bulk_wait_read(); // the store before has read the buffer
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                *reinterpret_cast<uint4*>(mine + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_uint4(h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0 && w.x0 + c0 < W) {
                                tma_store_4d(&map, mine, w.x0 + c0, w.y0 + row, m0 + l, w.f);
                                bulk_commit();
                            }
                        }
                    }
                } else {
                    __half* out = p.gcoef + ((int64_t)w.f * p.planes + m0) * HW + pix;
                    for (int l0 = 0; l0 < nr; l0 += 16) {
                        float acc[16];
                        tmem_ld_x16(at + l0, acc);
                        tmem_ld_wait();
                        if (inside) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                if (l0 + i < nr) {
                                    const float back = sback[m0 + l0 + i];
                                    *out = __float2half_rn(back != 0.f ? acc[i] * (back * ts.unscale) : 0.f);
                                    out += HW;
                                }
                            }
                        }
                    }
                }
            }
            return true;
        };
        bool go = true;                          // the group's: a thread leaves only where all do
        int started = -1;                        // row whose product is under way while the next row's G is computed
        for (int row = grp; row < w.rows; row += kGroups) {
            float v[G::kk];
            patch_grad<K>(s.U + row * G::UW + x, p.g.uh * G::UW, s.g + row * C * kGroupThreads + x, C, ts.scale, v, [] {});
            if (started >= 0 && !(go = finish(started))) break;
            if (ATOMS && !p.own_out) {           // every warp's stores have read the tile
                if (lane == 0) bulk_wait_read();
                ok = group_barrier_and(1 + grp, ok);
            }
            write_row<K>(sG, 128 * 128, x, v);
            fence_proxy_async_smem();
            tc_fence_before_sync();
            if (!(go = group_barrier_and(1 + grp, ok))) break;
            if (leads && elect_one()) multiply(0);
            __syncwarp();
            started = row;
        }
        if (go && started >= 0) go = finish(started);
        ok = ok && go;
        tc_fence_before_sync();
    }
    // ---- teardown: every product finished before tensor memory is freed, every store before shared memory is
    if (ATOMS && lane == 0) bulk_wait_all();
    __syncwarp();
    if (leads && elect_one()) { mma_commit(&ctl.drain); mbar_wait_drain(&ctl.drain, 0); }        // (the lane that issued them)
    __syncwarp();
    cp_async_wait_all_();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (ctl.wait.abort_flag && tid == 0) atomicExch(p.status, SR_ERR_TIMEOUT);
    if (warp == 0) tmem_dealloc(ctl.tmem_base, kGroups * 128);
}

// ---- gradient of the dictionary --------------------------------------------------------------------------------------------

// The second product. Rows of a block's tile are accumulated in tensor memory and added to registers (lane = atom) once a tile, where
// the scale changes and so that the tensor core's additions, which cut off, stay few.
template <int K, int MB>
__global__ void __launch_bounds__(kThreads, MB == 1 ? 2 : 1)
grad_dict_tc_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ GradTcParams p)
{
    using G = GGeo<K>;
    constexpr int TMEM_COLS = kGroups * MB * G::NB;
    extern __shared__ uint8_t smem_raw[];
    __shared__ GradCtl ctl;
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const Problem& pb = p.g.pb;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), grp = warp / (kGroupThreads / 32), x = tid % kGroupThreads, lane = tid & 31;
    const bool leads = warp % (kGroupThreads / 32) == 0;         // the group's first warp: its elected lane issues what one thread issues
    const int C = pb.c, D = pb.D, W = pb.W, s_ = pb.s;
    uint8_t* sG = smem + grp * G::G_BYTES;
    uint8_t* sPhi = smem + kGroups * G::G_BYTES + grp * p.stage_bytes;         // [64-pixel chunk][plane][128 B]
    // (the product reads 128 MB rows of a chunk, whatever lies there: they end in accumulators that nobody reads)
    const Floats s = carve_floats(smem + kGroups * G::G_BYTES + kGroups * p.stage_bytes, p, G::UW);

    init_ctl(ctl, p, tid);
    for (int i = tid; i < kGroups * (G::G_BYTES + p.stage_bytes) / 16; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    for (int i = tid; i < p.g.pb.c * p.g.trows * p.g.tcols + 8; i += kThreads) s.L[i] = 0.f;
    if (p.mode == kModeGlobal && tid < s_) ctl.atoms[tid] = (uint8_t)min((int)__ldg(p.idx + tid), D - 1);
    if (tid == 0 && p.tma) prefetch_tensormap(&map);
    fence_proxy_async_smem();
    if (warp == 0) tmem_alloc(&ctl.tmem_base, TMEM_COLS);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = ctl.tmem_base + grp * MB * G::NB;
    volatile WaitCtx* wc = &ctl.wait;
    const int64_t HW = (int64_t)pb.H * W;
    TileState<K> ts;
    ts.start(p, s.L, tid);
    const uint64_t g_desc = make_smem_desc(smem_u32(sG), 128 * 128, 1024, kSwizzle128B);
    const uint64_t a_desc = make_smem_desc(smem_u32(sPhi), 16, 1024, kSwizzle128B);
    constexpr uint32_t idesc = make_idesc_f16(128, G::NB, false, true);
    float total[MB][G::kk];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < G::kk; ++j) total[m][j] = 0.f;

    bool lose = p.lose != 0 && blockIdx.x == 0 && warp == 0;
    uint32_t phase = 0, fphase = 0;
    bool in_work = false;                        // a product of this group whose end has not been waited for
    bool landing = false;                        // (the group's first warp) a copy that has not been waited for
    bool ok = true;
    int parity = 0;
    uint8_t* chunk = sPhi + (x >> 6) * p.chunk_bytes;
    const int unit = (x & 63) >> 3, at2 = (x & 7) * 2;                         // this pixel's 16-byte unit and place in it
    auto place = [&](int l) { return reinterpret_cast<__half*>(chunk + l * 128 + ((unit ^ (l & 7)) << 4) + at2); };
    for (int t = blockIdx.x; t < p.g.num_tiles; t += gridDim.x, parity ^= 1) {
        const LrWindow w = ts.w;
        auto fetch = [&](int row) {              // the group's first warp: two boxes, bytes counted on full
            landing = true;
            if (!elect_one()) return;
            mbar_arrive_expect_tx(&ctl.full[grp], (uint32_t)p.rows * 256u);
            tma_load_4d(sPhi, &map, &ctl.full[grp], w.x0, w.y0 + row, 0, w.f);
            tma_load_4d(sPhi + p.chunk_bytes, &map, &ctl.full[grp], w.x0 + 64, w.y0 + row, 0, w.f);
        };
        if (p.tma && leads && grp < w.rows && ok) fetch(grp);                  // (the tile before was waited for at its end)
        __syncwarp();
        if (!(ok = ts.make(p, ctl, t, parity, s.L, s.V, s.U, s.g, tid, ok))) break;
        const bool inside = w.x0 + x < W;
        for (int row = grp; row < w.rows; row += kGroups) {
            float v[G::kk];
            patch_grad<K>(s.U + row * G::UW + x, p.g.uh * G::UW, s.g + row * C * kGroupThreads + x, C, ts.scale, v, [&] {
                // by now the row before has been multiplied: its stage takes this row's coefficients while G is being computed
                if (p.tma && in_work) {
                    if (leads) {
                        ok = __all_sync(0xffffffffu, ok && mbar_wait_short(&ctl.mma[grp], phase, wc));
                        if (ok) fetch(row);
                    }
                    __syncwarp();
                }
            });
            if (in_work) {
                ok = __all_sync(0xffffffffu, ok && mbar_wait_short(&ctl.mma[grp], phase, wc));
                phase ^= 1;
                in_work = false;
            }
            if (!inside) {
#pragma unroll
                for (int j = 0; j < G::kk; ++j) v[j] = 0.f;                    // (patches of columns beyond the image may be anything)
            }
            if (ok) write_row<K>(sG, 128 * 128, x, v);
            const int64_t pix = (int64_t)(w.y0 + row) * W + w.x0 + x;
            if (!p.tma && ok) {
                if (p.mode == kModeIdx || p.mode == kModeCompact) {
                    // the atoms that the pixel listed a row ago are cleared by the thread that wrote them (below)
                    if (inside)
                        for (int q = 0; q < s_; ++q) {
                            const int a = min((int)__ldg(p.idx + ((int64_t)w.f * s_ + q) * HW + pix), D - 1);
                            *place(a) = __ldg(p.coef + (p.mode == kModeCompact ? (int64_t)w.f * s_ + q : (int64_t)w.f * D + a) * HW + pix);
                        }
                } else {
                    const bool gather = p.mode == kModeGlobal && !(pb.flags & SR_COEF_COMPACT);
                    const __half* src = p.coef + (int64_t)w.f * p.planes * HW + pix;
                    for (int l0 = 0; l0 < p.rows; l0 += 16) {
                        __half h[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            h[i] = inside && l0 + i < p.rows ? __ldg(src + (int64_t)(gather ? ctl.atoms[l0 + i] : l0 + i) * HW) : __ushort_as_half(0);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (l0 + i < p.rows) *place(l0 + i) = h[i];
                    }
                }
            }
            fence_proxy_async_smem();
            tc_fence_before_sync();
            if (!(ok = group_barrier_and(1 + grp, ok))) break;
            if (leads) {
                bool there = true;
                if (p.tma) { there = __all_sync(0xffffffffu, mbar_wait_short(&ctl.full[grp], fphase, wc)); landing = !there; }
                if (there && elect_one()) {
                    tc_fence_after_sync();
#pragma unroll
                    for (int m = 0; m < MB; ++m) {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks) {
                            const uint64_t ad = a_desc + (uint64_t)((uint32_t)(m * 128 * 128 + (ks >> 2) * p.chunk_bytes + (ks & 3) * 32) >> 4);
                            mma_f16_ss(tmem + m * G::NB, ad, g_desc + (uint64_t)(ks * 2048 >> 4), idesc, row > grp || ks > 0);
                        }
                    }
                    if (!lose) mma_commit(&ctl.mma[grp]);
                }
                lose = false;
            }
            fphase ^= 1;
            in_work = true;
            __syncwarp();
            if (p.mode == kModeIdx || p.mode == kModeCompact) {
                // the stage goes back to zeros, which needs the product's end
                ok = __all_sync(0xffffffffu, mbar_wait_short(&ctl.mma[grp], phase, wc));
                phase ^= 1;
                in_work = false;
                if (inside && ok)
                    for (int q = 0; q < s_; ++q)
                        *place(min((int)__ldg(p.idx + ((int64_t)w.f * s_ + q) * HW + pix), D - 1)) = __ushort_as_half(0);
            }
        }
        if (!ok) continue;                       // (the next tile's barrier, or the end, tells the block)
        if (grp < w.rows) {
            if (in_work) {
                ok = __all_sync(0xffffffffu, mbar_wait_short(&ctl.mma[grp], phase, wc));
                phase ^= 1;
                in_work = false;
            }
            tc_fence_after_sync();
            if (ok) {
#pragma unroll
                for (int m = 0; m < MB; ++m) {
                    const uint32_t at = tmem + m * G::NB + ((uint32_t)(32 * (warp & 3)) << 16);
                    constexpr int STEP = 16;
#pragma unroll
                    for (int j0 = 0; j0 < G::kk; j0 += STEP) {
                        float hi[STEP], lo[STEP];
                        tmem_ld_x16(at + j0, hi);
                        tmem_ld_x16(at + G::LO_COL + j0, lo);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < STEP; ++i)
                            if (j0 + i < G::kk) total[m][j0 + i < G::kk ? j0 + i : 0] = fmaf(hi[i] + lo[i], ts.unscale, total[m][j0 + i < G::kk ? j0 + i : 0]);
                    }
                }
            }
            tc_fence_before_sync();
        }
    }
    // ---- teardown
    __syncwarp();
    if (leads && elect_one()) {                  // (the lane that issued copies and products)
        if (landing) mbar_wait_drain(&ctl.full[grp], fphase);
        mma_commit(&ctl.drain);
        mbar_wait_drain(&ctl.drain, 0);
    }
    __syncwarp();
    cp_async_wait_all_();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (ctl.wait.abort_flag && tid == 0) atomicExch(p.status, SR_ERR_TIMEOUT);
    if (warp == 0) tmem_dealloc(ctl.tmem_base, TMEM_COLS);
    // the two groups' sums, in their order, through shared memory (the operand tiles are done with)
    float* sum = reinterpret_cast<float*>(smem);
    float* out = p.partial + (int64_t)blockIdx.x * p.rows * G::kk;
    for (int gsel = kGroups - 1; gsel >= 0; --gsel) {
        if (grp == gsel) {
#pragma unroll
            for (int m = 0; m < MB; ++m) {
                const int l = m * 128 + 32 * (warp & 3) + lane;
                if (l < p.rows) {
#pragma unroll
                    for (int j = 0; j < G::kk; ++j) {
                        if (gsel == kGroups - 1) sum[l * G::kk + j] = total[m][j];
                        else out[l * G::kk + j] = total[m][j] + sum[l * G::kk + j];
                    }
                }
            }
        }
        __syncthreads();
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
        return (EncodeTiledFn)f;
    }();
    return fn;
}

int smem_optin()
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
int tile_rows(const Problem& pb)
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

template <typename Kern> cudaError_t allow_smem(Kern kern, bool (&done)[64])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!done[dev]) {
        if (cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_optin() - kStaticReserve)) return e;
        done[dev] = true;
    }
    return cudaSuccess;
}

// Blocks that fit a multiprocessor together (two at most: tensor memory, registers).
int blocks_per_sm(size_t smem) { return 2 * (smem + kStaticReserve) <= (size_t)smem_optin() ? 2 : 1; }

int coef_rows(const GradArgs& a) { return a.mode == kModeGlobal && (a.pb.flags & SR_COEF_COMPACT) ? a.pb.s : a.pb.D; }

// A [n][planes][H][W] binary16 tensor in boxes of 64 pixels of one row by `box_planes` planes, 128-byte swizzle.
bool encode_planes(CUtensorMap* map, const void* base, const Problem& pb, int planes, int box_planes)
{
    const cuuint64_t dims[4] = {(cuuint64_t)pb.W, (cuuint64_t)pb.H, (cuuint64_t)planes, (cuuint64_t)pb.n};
    const cuuint64_t strides[3] = {(cuuint64_t)pb.W * 2, (cuuint64_t)pb.W * pb.H * 2, (cuuint64_t)pb.W * pb.H * 2 * planes};
    const cuuint32_t es[4] = {1, 1, 1, 1}, box[4] = {64, 1, (cuuint32_t)box_planes, 1};
    return encode_fn() && encode_fn()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
                                      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Plane rows that TMA can store.
bool coef_atoms(const GradArgs& a) { return a.pb.W % 8 == 0 && ((uintptr_t)a.gcoef & 15) == 0 && encode_fn(); }

// own_out: bytes of a group's buffer for results. More than 128 atoms need one (the next product of the row reads G still); others
// have one where two blocks fit a multiprocessor with it.
template <int K> size_t coef_smem(Geom& g, const GradArgs& a, int* own_out)
{
    const int rows_pad = (coef_rows(a) + 15) & ~15;
    const size_t before = 1024 + kGroups * GGeo<K>::G_BYTES;
    const size_t rest = before + (size_t)GGeo<K>::BLOCKS * rows_pad * 128 + float_bytes<K>(g, a.pb, a.lr);
    const int buffer = (rows_pad < 128 ? (rows_pad + 31) / 32 : 4) * (kOutBytes / 4);
    *own_out = coef_atoms(a) && (rows_pad > 128 || blocks_per_sm(rest + kGroups * buffer) == 2) ? buffer : 0;
    const size_t all = rest + kGroups * *own_out;
    // atoms as rows: the product reads them 128 at a time, whatever lies behind the last one must be shared memory
    const size_t reach = before + (size_t)(GGeo<K>::BLOCKS - 1) * rows_pad * 128 + (size_t)((rows_pad + 127) / 128) * 128 * 128;
    return all > reach ? all : reach;
}

int stage_bytes_of(int rows) { return 2 * ((rows + 7) & ~7) * 128; }

template <int K> size_t dict_smem(Geom& g, const GradArgs& a)
{
    const int rows = grad_rows(a), mb = rows > 128 ? 2 : 1;
    // what the last chunk's 128 mb rows may reach must be shared memory
    const size_t operands = kGroups * ((size_t)GGeo<K>::G_BYTES + stage_bytes_of(rows));
    const size_t all = 1024 + operands + float_bytes<K>(g, a.pb, a.lr);
    const size_t reach = 1024 + operands - stage_bytes_of(rows) / 2 + (size_t)mb * 128 * 128;
    const size_t sums = 1024 + (size_t)rows * GGeo<K>::kk * sizeof(float);
    return all > reach ? (all > sums ? all : sums) : (reach > sums ? reach : sums);
}

GradTcParams common_params(const GradArgs& a)
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

template <int K, bool ATOMS> cudaError_t launch_coef_ka(const GradArgs& a)
{
    GradTcParams p = common_params(a);
    if (!p.status) return cudaErrorUnknown;
    const size_t smem = coef_smem<K>(p.g, a, &p.own_out);
    p.rows = coef_rows(a);
    CUtensorMap map{};
    if (ATOMS && !encode_planes(&map, a.gcoef, a.pb, p.planes, 32)) return cudaErrorUnknown;
    static bool done[64] = {false};
    if (cudaError_t e = allow_smem(grad_coef_tc_kernel<K, ATOMS>, done)) return e;
    const int most = sm_count() * blocks_per_sm(smem);
    grad_coef_tc_kernel<K, ATOMS><<<p.g.num_tiles < most ? p.g.num_tiles : most, kThreads, smem, a.st>>>(map, p);
    count_launches(1);
    return cudaGetLastError();
}

template <int K> cudaError_t launch_coef_k(const GradArgs& a) { return coef_atoms(a) ? launch_coef_ka<K, true>(a) : launch_coef_ka<K, false>(a); }

template <int K, int MB> cudaError_t launch_dict_km(const GradArgs& a, int* slots)
{
    GradTcParams p = common_params(a);
    if (!p.status) return cudaErrorUnknown;
    const size_t smem = dict_smem<K>(p.g, a);
    p.rows = grad_rows(a);
    p.stage_bytes = stage_bytes_of(p.rows);
    p.chunk_bytes = p.stage_bytes / 2;
    CUtensorMap map{};
    const Problem& pb = a.pb;
    const bool whole = a.mode == kModeDense || (a.mode == kModeGlobal && (pb.flags & SR_COEF_COMPACT));
    p.tma = whole && pb.W % 8 == 0 && ((uintptr_t)a.coef & 15) == 0 && encode_planes(&map, a.coef, pb, p.planes, p.rows);
    static bool done[64] = {false};
    if (cudaError_t e = allow_smem(grad_dict_tc_kernel<K, MB>, done)) return e;
    const int most = sm_count() * (MB == 1 ? blocks_per_sm(smem) : 1);
    const int blocks = p.g.num_tiles < most ? p.g.num_tiles : most;
    grad_dict_tc_kernel<K, MB><<<blocks, kThreads, smem, a.st>>>(map, p);
    count_launches(1);
    *slots = blocks;
    return cudaGetLastError();
}

template <int K> cudaError_t launch_dict_k(const GradArgs& a, int* slots)
{
    return grad_rows(a) > 128 ? launch_dict_km<K, 2>(a, slots) : launch_dict_km<K, 1>(a, slots);
}

bool form_supported(const GradArgs& a)
{
    const Problem& pb = a.pb;
    return a.coef_dtype == SR_F16 && (pb.k == 3 || pb.k == 5 || pb.k == 7) && pb.c <= kMaxC && smem_optin() > 0 &&
           (int64_t)((pb.W + TW - 1) / TW) * ((pb.H + 1) / 2) * pb.n <= 0x7FFFFFFF;
}

bool fits(size_t smem) { return smem + kStaticReserve <= (size_t)smem_optin(); }

} // namespace

bool grad_coef_tc_supported(const GradArgs& a)
{
    if (!form_supported(a) || a.mode == kModeIdx || a.mode == kModeCompact) return false;
    Geom g;
    int own_out;
    switch (a.pb.k) {
    case 3: return fits(coef_smem<3>(g, a, &own_out));
    case 5: return fits(coef_smem<5>(g, a, &own_out));
    default: return fits(coef_smem<7>(g, a, &own_out));
    }
}

bool grad_dict_tc_supported(const GradArgs& a)
{
    if (!form_supported(a)) return false;
    Geom g;
    switch (a.pb.k) {
    case 3: return fits(dict_smem<3>(g, a));
    case 5: return fits(dict_smem<5>(g, a));
    default: return fits(dict_smem<7>(g, a));
    }
}

cudaError_t launch_grad_coef_tc(const GradArgs& a)
{
    switch (a.pb.k) {
    case 3: return launch_coef_k<3>(a);
    case 5: return launch_coef_k<5>(a);
    default: return launch_coef_k<7>(a);
    }
}

cudaError_t launch_grad_dict_tc(const GradArgs& a, int* slots)
{
    switch (a.pb.k) {
    case 3: return launch_dict_k<3>(a, slots);
    case 5: return launch_dict_k<5>(a, slots);
    default: return launch_dict_k<7>(a, slots);
    }
}

} // namespace sr
