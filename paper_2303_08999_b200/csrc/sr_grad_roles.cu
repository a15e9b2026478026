// Both gradients of the dictionary regression in one kernel of specialised warps, for binary16 coefficients with at most 128 atoms:
// k in {3, 5, 7}, up to four channels, any width and every mode. (sr_grad_tc.cu: the mathematics, and more atoms.)
//
// What bounds a kernel whose warps do everything in turn is not the tensor core or memory but the waits between the steps of a row
// (1080p x4, D = 72, k = 5: 129 + 129 us in two kernels, 34 of each the up-sampled tile, against 95 us of traffic). Here one block per
// multiprocessor holds a pipeline, and G, which costs most, is computed once for both products:
//   G warps (kFG groups of four)   the up-sampled tile; G of every row, hi + lo, into a ring of tiles         g_full
//   load warps (three)             the row's coefficients into a ring of stages: TMA boxes, or (widths and    p_full
//                                  addresses TMA does not take, gathered planes, lists) a pixel a thread
//   MMA warp                       both products of a row; a row's filters in one of two accumulators         c_full, g_empty, p_empty
//                                  (lane = atom, column = pixel), the dictionary's sums over the tile in      d_full
//                                  one of two more
//   result warps (four)            a row's coefficient gradients to memory (c_empty), the tile's dictionary sums to registers (d_empty)
// Rows are numbered through the block's tiles; row i goes to G group i mod kFG, ring entries i mod their count, accumulator i mod 2.
// Every wait is bounded: on expiry a warp raises the block's flag and leaves its loop, as every other does at its next wait.
#include "sr_grad_tc.cuh"

namespace sr {

namespace {

using namespace ptx;
using namespace tile;
using namespace gradtc;

constexpr int kFG = 2;                                       // groups of G warps
// Sixteen warps, so that each has 128 registers; the result warps start at a multiple of four (their share of tensor memory).
constexpr int kResultWarp = kFG * 4, kLoadWarp = kResultWarp + 4, kMmaWarp = kLoadWarp + 3;
constexpr int kRoleThreads = (kMmaWarp + 1) * 32, kLoadThreads = 96;
static_assert(kRoleThreads == 512, "128 registers a thread");
constexpr int kMaxG = 4, kMaxP = 4, kUnscales = 16;
template <int K> constexpr int kRing = K == 7 ? 2 : kMaxG;      // G tiles (those of 7 x 7 are twice as large)

struct __align__(16) RoleCtl {
    GradCtl c;                                               // (its mma / full barriers are not used)
    uint64_t g_full[kMaxG], g_empty[kMaxG], p_full[kMaxP], p_empty[kMaxP];
    uint64_t c_full[2], c_empty[2], d_full[2], d_empty[2];
    float unscale[kUnscales];                                // of the tiles, by number
    float back[128];                                         // 2^e of each plane's atom (0: a plane outside the subset)
    uint32_t listed[128][4];                                 // lists: the row's pixels that list the atom
};

struct RoleParams {
    GradTcParams b;
    int atoms;                   // rows of the first product: D, or s of a compact subset
    int planes_in, planes_out;   // of a frame in coef and gcoef
    int p_stages;
    int tma_in, tma_out;
    int want_coef, want_dict;
};

template <int K> struct RoleSmem {
    uint8_t *G, *D, *out, *Phi;
    Floats f;
};
// [G ring][atoms][results][coefficient ring][floats]
template <int K> __device__ __forceinline__ RoleSmem<K> carve(uint8_t* at, const RoleParams& p)
{
    RoleSmem<K> s;
    s.G = at;
    s.D = s.G + kRing<K> * GGeo<K>::G_BYTES;
    s.out = s.D + (p.want_coef ? GGeo<K>::BLOCKS * 128 * 128 : 0);
    s.Phi = s.out + (p.want_coef ? 2 * kOutBytes : 0);
    s.f = carve_floats(s.Phi + p.p_stages * p.b.stage_bytes, p.b, GGeo<K>::UW);
    return s;
}

__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile WaitCtx* wc, bool ok)
{
    return __all_sync(0xffffffffu, ok && mbar_wait_short(bar, parity, wc));
}

// The tiles of the block, in every role's own steps.
struct Tiles {
    int t, base, n;                                          // tile, number of its first row, number of the tile
    int f, y0, x0, rows;
    __device__ __forceinline__ explicit Tiles(const Geom& g) : t(blockIdx.x), base(0), n(0) { if (more(g)) decode_tile(g, t, f, y0, x0, rows); }
    __device__ __forceinline__ bool more(const Geom& g) const { return t < g.num_tiles; }
    __device__ __forceinline__ void next(const Geom& g)
    {
        base += rows;
        ++n;
        t += gridDim.x;
        if (more(g)) decode_tile(g, t, f, y0, x0, rows);
    }
};

// ---- G warps ----------------------------------------------------------------------------------------------------------------

template <int K> __device__ __forceinline__ bool g_role(const RoleParams& p, RoleCtl& ctl, const RoleSmem<K>& s, int tid)
{
    using G = GGeo<K>;
    const int grp = __shfl_sync(0xffffffffu, tid >> 5, 0) / 4, x = tid % kGroupThreads, C = p.b.g.pb.c;
    volatile WaitCtx* wc = &ctl.c.wait;
    TileState<K, kFG, true> ts;
    Tiles tl(p.b.g);
    ts.start(p.b, s.f, tid, grp);                            // (row `grp` is the group's first of the block)
    bool ok = true;
    int parity = 0;
    for (; tl.more(p.b.g); parity ^= 1) {
        const int first = (grp + kFG - tl.base % kFG) % kFG;             // the group's first row of the tile
        Tiles after = tl;
        after.next(p.b.g);
        const int next_first = (grp + kFG - after.base % kFG) % kFG;
        if (!(ok = ts.make(p.b, ctl.c, tl.t, parity, s.f, tid, ok, first, next_first, &ctl.unscale[tl.n % kUnscales]))) break;
        const bool inside = tl.x0 + x < p.b.g.pb.W;
        for (int row = first; row < tl.rows; row += kFG) {
            float v[G::kk];
            patch_grad<K>(s.f.U + row * G::UW + x, p.b.g.uh * G::UW, s.f.g + row * C * kGroupThreads + x, C, ts.scale, v, [] {});
            if (!inside) {
#pragma unroll
                for (int j = 0; j < G::kk; ++j) v[j] = 0.f;              // (patches of columns beyond the image may be anything)
            }
            const int item = tl.base + row, st = item % kRing<K>;
            ok = wait_all(&ctl.g_empty[st], ((item / kRing<K>) & 1) ^ 1, wc, ok);
            if (ok) write_row<K>(s.G + st * G::G_BYTES, 128 * 128, x, v);
            fence_proxy_async_smem();
            mbar_arrive(&ctl.g_full[st]);
        }
        tl = after;
    }
    cp_async_wait_all_();
    return ok;
}

__device__ __forceinline__ bool load_barrier_and(bool ok)
{
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 3, %2, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((int)ok), "n"(kLoadThreads) : "memory");
    return r != 0;
}

// ---- load warps ---------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void load_role(const CUtensorMap* map, const RoleParams& p, RoleCtl& ctl, uint8_t* sPhi, int tid)
{
    const Problem& pb = p.b.g.pb;
    volatile WaitCtx* wc = &ctl.c.wait;
    const int64_t HW = (int64_t)pb.H * pb.W;
    if (p.tma_in) {
        // one lane: two boxes a row, bytes counted on the stage's barrier
        if ((tid >> 5) != 0 || !elect_one()) return;
        bool ok = true;
        int issued = 0;
        for (Tiles tl(p.b.g); tl.more(p.b.g) && ok; tl.next(p.b.g))
            for (int row = 0; row < tl.rows; ++row) {
                const int item = tl.base + row, st = item % p.p_stages;
                if (!(ok = mbar_wait_short(&ctl.p_empty[st], ((item / p.p_stages) & 1) ^ 1, wc))) break;
                uint8_t* dst = sPhi + st * p.b.stage_bytes;
                mbar_arrive_expect_tx(&ctl.p_full[st], (uint32_t)p.b.rows * 256u);
                tma_load_4d(dst, map, &ctl.p_full[st], tl.x0, tl.y0 + row, 0, tl.f);
                tma_load_4d(dst + p.b.chunk_bytes, map, &ctl.p_full[st], tl.x0 + 64, tl.y0 + row, 0, tl.f);
                issued = item + 1;
            }
        // what was asked for lands before shared memory is given up
        for (int item = issued > p.p_stages ? issued - p.p_stages : 0; item < issued; ++item)
            mbar_wait_drain(&ctl.p_full[item % p.p_stages], (item / p.p_stages) & 1);
        return;
    }
    const int s = pb.s;
    const bool lists = p.b.mode == kModeIdx || p.b.mode == kModeCompact;
    const bool gather = p.b.mode == kModeGlobal && !(pb.flags & SR_COEF_COMPACT);
    const __half zero = __ushort_as_half(0);
    bool ok = true;
    for (Tiles tl(p.b.g); tl.more(p.b.g); tl.next(p.b.g)) {
        for (int row = 0; row < tl.rows; ++row) {
            const int item = tl.base + row, st = item % p.p_stages;
            uint8_t* stage = sPhi + st * p.b.stage_bytes;
            ok = wait_all(&ctl.p_empty[st], ((item / p.p_stages) & 1) ^ 1, wc, ok);
            if (lists) {
                if (ok)
                    for (int i = tid; i < p.b.stage_bytes / 16; i += kLoadThreads) reinterpret_cast<uint4*>(stage)[i] = make_uint4(0, 0, 0, 0);
                ok = load_barrier_and(ok);                               // (the load warps leave together: they meet here)
            }
            if (!ok) return;
            for (int x = tid; x < 128; x += kLoadThreads) {
                const bool inside = tl.x0 + x < pb.W;
                uint8_t* chunk = stage + (x >> 6) * p.b.chunk_bytes;
                const int unit = (x & 63) >> 3, at2 = (x & 7) * 2;       // this pixel's 16-byte unit and place in it
                auto place = [&](int l) { return reinterpret_cast<__half*>(chunk + l * 128 + ((unit ^ (l & 7)) << 4) + at2); };
                const int64_t pix = (int64_t)(tl.y0 + row) * pb.W + tl.x0 + x;
                const __half* src = p.b.coef + (int64_t)tl.f * p.planes_in * HW + pix;
                if (lists) {
                    const uint8_t* list = p.b.idx + (int64_t)tl.f * s * HW + pix;
                    for (int q0 = 0; inside && q0 < s; q0 += 8) {
                        int a[8];
                        __half v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) a[i] = q0 + i < s ? min((int)__ldg(list + (int64_t)(q0 + i) * HW), pb.D - 1) : 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = q0 + i < s ? __ldg(src + (int64_t)(p.b.mode == kModeCompact ? q0 + i : a[i]) * HW) : zero;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (q0 + i < s) *place(a[i]) = v[i];
                    }
                } else {
                    for (int l0 = 0; l0 < p.b.rows; l0 += 24) {
                        __half h[24];
#pragma unroll
                        for (int i = 0; i < 24; ++i)
                            h[i] = inside && l0 + i < p.b.rows ? __ldg(src + (int64_t)(gather ? ctl.c.atoms[l0 + i] : l0 + i) * HW) : zero;
#pragma unroll
                        for (int i = 0; i < 24; ++i)
                            if (l0 + i < p.b.rows) *place(l0 + i) = h[i];
                    }
                }
            }
            fence_proxy_async_smem();
            mbar_arrive(&ctl.p_full[st]);
        }
    }
}

// ---- MMA warp -----------------------------------------------------------------------------------------------------------------

template <int K> __device__ __forceinline__ void mma_role(const RoleParams& p, RoleCtl& ctl, const RoleSmem<K>& s, uint32_t tmem)
{
    using G = GGeo<K>;
    volatile WaitCtx* wc = &ctl.c.wait;
    const uint64_t g_desc0 = make_smem_desc(smem_u32(s.G), 16, 1024, kSwizzle128B);              // rows: K-major
    const uint64_t gt_desc0 = make_smem_desc(smem_u32(s.G), 128 * 128, 1024, kSwizzle128B);      // columns: MN-major
    const uint64_t d_desc = make_smem_desc(smem_u32(s.D), 16, 1024, kSwizzle128B);
    const uint64_t a_desc0 = make_smem_desc(smem_u32(s.Phi), 16, 1024, kSwizzle128B);
    constexpr uint32_t kGLo = (G::BLOCKS == 2 ? 128 * 128 : G::LO_CHUNK * 16) >> 4;
    constexpr uint32_t idesc_c = make_idesc_f16(128, 128, false, false), idesc_d = make_idesc_f16(128, G::NB, false, true);
    bool lose = p.b.lose != 0 && blockIdx.x == 0;
    bool ok = true;
    for (Tiles tl(p.b.g); tl.more(p.b.g) && ok; tl.next(p.b.g)) {
        const uint32_t d_acc = tmem + 256 + (tl.n & 1) * G::NB;
        for (int row = 0; row < tl.rows; ++row) {
            const int item = tl.base + row, gs = item % kRing<K>;
            if (p.want_coef) ok = wait_all(&ctl.c_empty[item & 1], ((item >> 1) & 1) ^ 1, wc, ok);
            if (p.want_dict && row == 0) ok = wait_all(&ctl.d_empty[tl.n & 1], ((tl.n >> 1) & 1) ^ 1, wc, ok);
            ok = wait_all(&ctl.g_full[gs], (item / kRing<K>) & 1, wc, ok);
            if (!ok) break;
            tc_fence_after_sync();
            const uint32_t g_off = (uint32_t)(gs * G::G_BYTES) >> 4;
            if (p.want_coef) {
                if (elect_one()) {
                    const uint32_t acc = tmem + (item & 1) * 128;
#pragma unroll
                    for (int ks = 0; ks < G::KSTEPS; ++ks) {
                        const uint64_t gh = g_desc0 + g_off + 2 * ks, dh = d_desc + 2 * ks;
                        mma_f16_ss(acc, dh, gh, idesc_c, ks > 0);
                        mma_f16_ss(acc, dh, gh + kGLo, idesc_c, 1u);
                        mma_f16_ss(acc, dh + kGLo, gh, idesc_c, 1u);
                    }
                    if (!lose) mma_commit(&ctl.c_full[item & 1]);
                }
                __syncwarp();
            }
            if (p.want_dict) {
                const int ps = item % p.p_stages;
                ok = wait_all(&ctl.p_full[ps], (item / p.p_stages) & 1, wc, ok);
                if (!ok) break;
                tc_fence_after_sync();
                if (elect_one()) {
                    const uint32_t a_off = (uint32_t)(ps * p.b.stage_bytes) >> 4, a_chunk = (uint32_t)p.b.chunk_bytes >> 4;
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        mma_f16_ss(d_acc, a_desc0 + a_off + (ks >> 2) * a_chunk + (ks & 3) * 2, gt_desc0 + g_off + (uint32_t)(ks * 2048 >> 4), idesc_d,
                                   row > 0 || ks > 0);
                    if (!(lose && !p.want_coef)) mma_commit(&ctl.p_empty[ps]);
                    if (row == tl.rows - 1) mma_commit(&ctl.d_full[tl.n & 1]);
                }
                __syncwarp();
            }
            if (elect_one()) mma_commit(&ctl.g_empty[gs]);
            __syncwarp();
            lose = false;
        }
    }
    // tensor memory is freed only once every product has finished
    if (elect_one()) { mma_commit(&ctl.c.drain); mbar_wait_drain(&ctl.c.drain, 0); }
    __syncwarp();
}

// ---- result warps ---------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ bool result_barrier(bool ok) { return group_barrier_and(2, ok); }

template <int K> __device__ __forceinline__ void result_role(const CUtensorMap* map, const RoleParams& p, RoleCtl& ctl, const RoleSmem<K>& s, uint32_t tmem, int tid)
{
    using G = GGeo<K>;
    const Problem& pb = p.b.g.pb;
    volatile WaitCtx* wc = &ctl.c.wait;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, l = 32 * warp + lane, W = pb.W;
    const int64_t HW = (int64_t)pb.H * W;
    const uint32_t at = tmem + ((uint32_t)(32 * warp) << 16);
    constexpr int STEP = K == 7 ? 16 : 32;                   // accumulator columns at a time (registers)
    const bool listed = p.b.mode == kModeIdx, compact = p.b.mode == kModeCompact;
    const bool together = p.want_coef && (listed || compact);        // these meet at barriers, so they leave together
    const bool mine = 32 * warp < p.atoms;                   // this warp has atoms
    const float back = p.want_coef && l < p.atoms ? ctl.back[l] : 0.f;
    float total[G::kk];
#pragma unroll
    for (int j = 0; j < G::kk; ++j) total[j] = 0.f;
    bool ok = true;
    int buffer = 0;
    for (Tiles tl(p.b.g); tl.more(p.b.g) && ok; tl.next(p.b.g)) {
        for (int row = 0; p.want_coef && row < tl.rows; ++row) {
            const int item = tl.base + row;
            const int64_t pix = (int64_t)(tl.y0 + row) * W + tl.x0;
            uint32_t keep[4] = {~0u, ~0u, ~0u, ~0u};
            if (listed) {                                    // which of the row's pixels list this lane's atom
                if (!(ok = result_barrier(ok))) break;       // the row before has been read
#pragma unroll
                for (int i = 0; i < 4; ++i) ctl.listed[tid][i] = 0u;
                if (!(ok = result_barrier(ok))) break;
                if (tl.x0 + tid < W)
                    for (int q = 0; q < pb.s; ++q) {
                        const int a = min((int)__ldg(p.b.idx + ((int64_t)tl.f * pb.s + q) * HW + pix + tid), pb.D - 1);
                        atomicOr(&ctl.listed[a][tid >> 5], 1u << (tid & 31));
                    }
            }
            ok = wait_all(&ctl.c_full[item & 1], (item >> 1) & 1, wc, ok);
            if (listed) {
                if (!(ok = result_barrier(ok))) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) keep[i] = ctl.listed[l][i];
            }
            tc_fence_after_sync();
            const float k = back * *(volatile float*)&ctl.unscale[tl.n % kUnscales];
#pragma unroll
            for (int c0 = 0; c0 < 128; c0 += 64) {
                uint32_t h[32];
                uint8_t* to = s.out + buffer * kOutBytes + warp * 4096;
                if (mine && ok) {
#pragma unroll
                    for (int c1 = 0; c1 < 64; c1 += STEP) {
                        float acc[STEP];
#pragma unroll
                        for (int i = 0; i < STEP; i += 16) tmem_ld_x16(at + (item & 1) * 128 + c0 + c1 + i, acc + i);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < STEP / 2; ++i) {
                            const __half2 v2 = __floats2half2_rn(acc[2 * i] * k, acc[2 * i + 1] * k);
                            h[c1 / 2 + i] = *reinterpret_cast<const uint32_t*>(&v2);
                        }
                    }
                    if (back == 0.f) {                       // outside the subset: zeros, whatever G is
#pragma unroll
                        for (int i = 0; i < 32; ++i) h[i] = 0u;
                    }
                    if (listed) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const uint32_t two = keep[(c0 + 2 * i) / 32] >> ((c0 + 2 * i) % 32);
                            h[i] &= ((two & 1u) ? 0xFFFFu : 0u) | ((two & 2u) ? 0xFFFF0000u : 0u);
                        }
                    }
                }
                if (c0 == 64) {                              // the accumulator has been read
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.c_empty[item & 1]);
                }
                if (compact) {
                    if (!(ok = result_barrier(ok))) break;   // the buffer's values two chunks ago have been taken
                } else {
                    if (lane == 0) bulk_wait_read_but_one(); // the store two chunks ago has read the buffer
                    __syncwarp();
                }
                if (mine && ok) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4*>(to + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_uint4(h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
                }
                if (compact) {
                    // values by rank: a pixel's listed atoms out of the chunk
                    if (!(ok = result_barrier(ok))) break;
                    const int px = tid & 63;
                    if (tl.x0 + c0 + px < W)
                        for (int q = tid >> 6; q < pb.s; q += 2) {
                            const int64_t pl = ((int64_t)tl.f * pb.s + q) * HW + pix + c0 + px;
                            const int a = min((int)__ldg(p.b.idx + pl), pb.D - 1);
                            p.b.gcoef[pl] = *reinterpret_cast<const __half*>(s.out + buffer * kOutBytes + (a >> 5) * 4096 + (a & 31) * 128 +
                                                                            ((((px >> 3) ^ (a & 7))) << 4) + (px & 7) * 2);
                        }
                } else if (p.tma_out) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0 && mine && ok && tl.x0 + c0 < W) tma_store_4d(map, to, tl.x0 + c0, tl.y0 + row, 32 * warp, tl.f);
                    if (lane == 0) bulk_commit();            // (an empty group where nothing was stored: groups are counted)
                } else if (mine && ok) {
                    // any alignment: a plane's 64 pixels a warp, two elements a lane
                    __syncwarp();
                    __half* dst = p.b.gcoef + ((int64_t)tl.f * p.planes_out + 32 * warp) * HW + pix + c0;
                    const int left = W - tl.x0 - c0, most = min(32, p.atoms - 32 * warp);
                    for (int a = 0; a < most; ++a, dst += HW) {
                        const uint8_t* from = to + a * 128;
                        const int p0 = lane, p1 = lane + 32;
                        if (p0 < left) dst[p0] = *reinterpret_cast<const __half*>(from + (((p0 >> 3) ^ (a & 7)) << 4) + (p0 & 7) * 2);
                        if (p1 < left) dst[p1] = *reinterpret_cast<const __half*>(from + (((p1 >> 3) ^ (a & 7)) << 4) + (p1 & 7) * 2);
                    }
                    __syncwarp();
                }
                buffer ^= 1;
            }
            if (!ok) break;
        }
        if (p.want_dict && ok) {
            ok = wait_all(&ctl.d_full[tl.n & 1], (tl.n >> 1) & 1, wc, ok);
            if (together) ok = result_barrier(ok);
            tc_fence_after_sync();
            if (!ok) break;
            const float un = *(volatile float*)&ctl.unscale[tl.n % kUnscales];
            if (32 * warp < p.b.rows) {
                const uint32_t d = at + 256 + (tl.n & 1) * G::NB;
#pragma unroll
                for (int j0 = 0; j0 < G::kk; j0 += 16) {
                    float hi[16], lo[16];
                    tmem_ld_x16(d + j0, hi);
                    tmem_ld_x16(d + G::LO_COL + j0, lo);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (j0 + i < G::kk) total[j0 + i < G::kk ? j0 + i : 0] = fmaf(hi[i] + lo[i], un, total[j0 + i < G::kk ? j0 + i : 0]);
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.d_empty[tl.n & 1]);
        }
    }
    if (lane == 0) bulk_wait_all();
    if (p.want_dict && l < p.b.rows) {
        float* out = p.b.partial + ((int64_t)blockIdx.x * p.b.rows + l) * G::kk;
#pragma unroll
        for (int j = 0; j < G::kk; ++j) out[j] = total[j];
    }
}

template <int K>
__global__ void __launch_bounds__(kRoleThreads, 1)
grad_roles_kernel(const __grid_constant__ CUtensorMap map_in, const __grid_constant__ CUtensorMap map_out, const __grid_constant__ RoleParams p)
{
    using G = GGeo<K>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ RoleCtl ctl;
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const RoleSmem<K> s = carve<K>(smem, p);
    const Problem& pb = p.b.g.pb;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), D = pb.D;

    init_ctl(ctl.c, p.b, tid, kRoleThreads, 1);
    if (tid == 0) {
        for (int i = 0; i < kMaxG; ++i) { mbar_init(&ctl.g_full[i], kGroupThreads); mbar_init(&ctl.g_empty[i], 1); }
        for (int i = 0; i < kMaxP; ++i) { mbar_init(&ctl.p_full[i], p.tma_in ? 1 : kLoadThreads); mbar_init(&ctl.p_empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&ctl.c_full[i], 1); mbar_init(&ctl.c_empty[i], 4); mbar_init(&ctl.d_full[i], 1); mbar_init(&ctl.d_empty[i], 4); }
        fence_barrier_init();
        if (p.tma_in) prefetch_tensormap(&map_in);
        if (p.tma_out) prefetch_tensormap(&map_out);
    }
    // (what the products read beyond the atoms, planes and taps written ends in lanes and columns that nobody reads)
    for (int i = tid; i < pb.c * p.b.g.trows * p.b.g.tcols + 8; i += kRoleThreads) s.f.L[i] = 0.f;
    if (p.b.mode == kModeGlobal && tid < pb.s) ctl.c.atoms[tid] = (uint8_t)min((int)__ldg(p.b.idx + tid), D - 1);
    __syncthreads();
    if (p.want_coef)
        for (int q = tid; q < p.atoms; q += kRoleThreads) ctl.back[q] = write_atom<K>(p.b, s.D, 128 * 128, q);
    fence_proxy_async_smem();
    if (warp == kMmaWarp) tmem_alloc(&ctl.c.tmem_base, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = ctl.c.tmem_base;

    if (warp < kResultWarp) g_role<K>(p, ctl, s, tid);
    else if (warp < kLoadWarp) result_role<K>(&map_out, p, ctl, s, tmem, tid - kResultWarp * 32);
    else if (warp < kMmaWarp) { if (p.want_dict) load_role(&map_in, p, ctl, s.Phi, tid - kLoadWarp * 32); }
    else mma_role<K>(p, ctl, s, tmem);

    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (ctl.c.wait.abort_flag && tid == 0) atomicExch(p.b.status, SR_ERR_TIMEOUT);
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

// ---- host ------------------------------------------------------------------------------------------------------------------------

int out_planes(const GradArgs& a) { return a.mode == kModeCompact || (a.mode == kModeGlobal && (a.pb.flags & SR_COEF_COMPACT)) ? a.pb.s : a.pb.D; }
int product_atoms(const GradArgs& a) { return a.mode == kModeGlobal && (a.pb.flags & SR_COEF_COMPACT) ? a.pb.s : a.pb.D; }

// As many coefficient stages up to four as fit; at least two.
template <int K> bool plan(RoleParams& p, const GradArgs& a, size_t& smem)
{
    p.want_coef = a.gcoef != nullptr;
    p.want_dict = a.gdict || a.ggamma;
    p.atoms = product_atoms(a);
    p.b.rows = grad_rows(a);
    p.b.stage_bytes = stage_bytes_of(p.b.rows);
    p.b.chunk_bytes = p.b.stage_bytes / 2;
    const size_t floats = float_bytes<K>(p.b.g, a.pb, a.lr);
    const size_t fixed = 1024 + (size_t)kRing<K> * GGeo<K>::G_BYTES + (p.want_coef ? GGeo<K>::BLOCKS * 128 * 128 + 2 * kOutBytes : 0) + floats;
    p.p_stages = 0;
    smem = fixed;
    if (p.want_dict) {
        for (p.p_stages = kMaxP; p.p_stages >= 2; --p.p_stages) {
            smem = fixed + (size_t)p.p_stages * p.b.stage_bytes;
            // the second product reads 128 rows of a chunk, whatever lies behind the last one must be shared memory
            const size_t reach = smem - floats - p.b.chunk_bytes + 128 * 128;
            if (smem < reach) smem = reach;
            if (fits(smem)) break;
        }
        if (p.p_stages < 2) return false;
    }
    return fits(smem);
}

template <int K> cudaError_t launch_k(const GradArgs& a, int* slots)
{
    RoleParams p{};
    p.b = common_params(a);
    if (!p.b.status) return cudaErrorUnknown;
    size_t smem = 0;
    if (!plan<K>(p, a, smem)) return cudaErrorNotSupported;
    p.planes_out = out_planes(a);
    p.planes_in = p.planes_out;
    CUtensorMap in{}, out{};
    const Problem& pb = a.pb;
    const bool whole = a.mode == kModeDense || (a.mode == kModeGlobal && (pb.flags & SR_COEF_COMPACT));
    if (p.want_dict && whole && pb.W % 8 == 0 && ((uintptr_t)a.coef & 15) == 0) p.tma_in = encode_planes(&in, a.coef, pb, p.planes_in, p.b.rows);
    if (p.want_coef && a.mode != kModeCompact && pb.W % 8 == 0 && ((uintptr_t)a.gcoef & 15) == 0) p.tma_out = encode_planes(&out, a.gcoef, pb, p.planes_out, 32);
    static bool done[64] = {false};
    if (cudaError_t e = allow_smem(grad_roles_kernel<K>, done)) return e;
    const int blocks = p.b.g.num_tiles < sm_count() ? p.b.g.num_tiles : sm_count();
    grad_roles_kernel<K><<<blocks, kRoleThreads, smem, a.st>>>(in, out, p);
    count_launches(1);
    *slots = blocks;
    return cudaGetLastError();
}

template <int K> bool plan_fits(const GradArgs& a)
{
    RoleParams p{};
    size_t smem;
    return plan<K>(p, a, smem);
}

} // namespace

bool grad_roles_supported(const GradArgs& a)
{
    if (!form_supported(a) || a.pb.D > 128) return false;
    switch (a.pb.k) {
    case 3: return plan_fits<3>(a);
    case 5: return plan_fits<5>(a);
    default: return plan_fits<7>(a);
    }
}

cudaError_t launch_grad_roles(const GradArgs& a, int* slots)
{
    switch (a.pb.k) {
    case 3: return launch_k<3>(a, slots);
    case 5: return launch_k<5>(a, slots);
    default: return launch_k<7>(a, slots);
    }
}

} // namespace sr
