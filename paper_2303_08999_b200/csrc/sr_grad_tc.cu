// Gradients of the dictionary regression on the tcgen05 tensor cores, for binary16 coefficients: k in {3, 5, 7}, up to four channels,
// any width and number of atoms. For what the one kernel of sr_grad_roles.cu does not take: more than 128 atoms, operands that leave
// it no room, odd widths with few planes.
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
#include "sr_grad_tc.cuh"

namespace sr {

namespace {

using namespace ptx;
using namespace tile;
using namespace gradtc;

constexpr int kThreads = 256, kGroups = 2;

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
    const int C = pb.c, W = pb.W, rows_pad = (p.rows + 15) & ~15;
    uint8_t* sG = smem + grp * G::G_BYTES;
    uint8_t* sD = smem + kGroups * G::G_BYTES;   // [column][rows_pad][128 B]
    const int d_block = rows_pad * 128;
    // results on their way out: behind the atoms (4 KB for each warp that has some), or in the G tile
    uint8_t* sOut = ATOMS && p.own_out ? sD + G::BLOCKS * d_block + grp * p.own_out : sG;
    const Floats s = carve_floats(sD + G::BLOCKS * d_block + (ATOMS ? kGroups * p.own_out : 0), p, G::UW);

    init_ctl(ctl, p, tid, kThreads, kGroups);
    for (int i = tid; i < (kGroups * G::G_BYTES + G::BLOCKS * d_block) / 16; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    for (int i = tid; i < p.g.pb.c * p.g.trows * p.g.tcols + 8; i += kThreads) s.L[i] = 0.f;
    __syncthreads();
    TileState<K, kGroups, false> ts;
    Tiles tl(p.g);
    ts.start(p, tl, s, tid, grp);
    for (int q = tid; q < p.rows; q += kThreads) sback[q] = write_atom<K>(p, sD, d_block, q);
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
    for (; tl.more(p.g); parity ^= 1) {
        tl.next(p.g);                            // (the tile after the one in work)
        const LrWindow w = ts.w;
        if (!(ok = ts.make(p, ctl, tl, parity, s, tid, ok, grp, grp, nullptr))) break;
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

    init_ctl(ctl, p, tid, kThreads, kGroups);
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
    TileState<K, kGroups, false> ts;
    Tiles tl(p.g);
    ts.start(p, tl, s, tid, grp);
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
    for (; tl.more(p.g); parity ^= 1) {
        tl.next(p.g);                            // (the tile after the one in work)
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
        if (!(ok = ts.make(p, ctl, tl, parity, s, tid, ok, grp, grp, nullptr))) break;
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
                    // (what a row put there is taken back by the thread that did, below)
                    const uint8_t* list = p.idx + (int64_t)w.f * s_ * HW + pix;
                    const __half* src = p.coef + (int64_t)w.f * p.planes * HW + pix;
                    for (int q0 = 0; inside && q0 < s_; q0 += 8) {       // (eight loads in flight)
                        int a[8];
                        __half h[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) a[i] = q0 + i < s_ ? min((int)__ldg(list + (int64_t)(q0 + i) * HW), D - 1) : 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i) h[i] = q0 + i < s_ ? __ldg(src + (int64_t)(p.mode == kModeCompact ? q0 + i : a[i]) * HW) : __ushort_as_half(0);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (q0 + i < s_) *place(a[i]) = h[i];
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
                const uint8_t* list = p.idx + (int64_t)w.f * s_ * HW + pix;
                for (int q0 = 0; inside && ok && q0 < s_; q0 += 8) {
                    int a[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) a[i] = q0 + i < s_ ? min((int)__ldg(list + (int64_t)(q0 + i) * HW), D - 1) : -1;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (a[i] >= 0) *place(a[i]) = __ushort_as_half(0);
                }
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

// Blocks that fit a multiprocessor together (two at most: tensor memory, registers).
int blocks_per_sm(size_t smem) { return 2 * (smem + kStaticReserve) <= (size_t)smem_optin() ? 2 : 1; }

int coef_rows(const GradArgs& a) { return a.mode == kModeGlobal && (a.pb.flags & SR_COEF_COMPACT) ? a.pb.s : a.pb.D; }

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
