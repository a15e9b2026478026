// Both gradients of the dictionary regression in one kernel of specialised warps, for binary16 coefficients with at most 128 atoms:
// k in {3, 5, 7}, up to four channels, any width and every mode. (sr_grad_tc.cu: the mathematics, and more atoms.)
//
// What bounds a kernel whose warps do everything in turn is not the tensor core or memory but the waits between the steps of a row
// (1080p x4, D = 72, k = 5: 129 + 129 us in two kernels, 34 of each the up-sampled tile, against 95 us of traffic). Here one block per
// multiprocessor holds a pipeline, and G, which costs most, is computed once for both products:
//   G warps (kFG groups of four)   the up-sampled tile; G of every row, hi + lo, into a ring of tiles         g_full
//   load warps (two)               the row's coefficients into a ring of stages: TMA boxes, or (widths and    p_full
//                                  addresses TMA does not take, gathered planes, lists) a pixel a thread
//   MMA warps (one a product)      a row's coefficient gradients in one of two accumulators (lane = atom,     c_full, g_empty
//                                  column = pixel), the dictionary's sums over the tile in one of two more     d_full, p_empty, g_empty
//   result warps (kRG groups of four)  a row's coefficient gradients to memory (c_empty), the tile's dictionary sums to registers (d_empty)
// Rows are numbered through the block's tiles; row i goes to G group i mod kFG, ring entries i mod their count, accumulator i mod 2.
// Waits suspend (mbar_wait): warps with time to spare must not take issue slots from those that set the pace.
// Every wait is bounded: on expiry a warp raises the block's flag and leaves its loop, as every other does at its next wait.
#include "sr_grad_tc.cuh"

namespace sr {

namespace {

using namespace ptx;
using namespace tile;
using namespace gradtc;

constexpr int kFG = 2;                                       // groups of G warps
constexpr int kRG = 2;                                       // groups of result warps: rows of one accumulator each
constexpr int kResultWarp = kFG * 4, kLoadWarp = kResultWarp + kRG * 4, kMmaWarp = kLoadWarp + 2;
constexpr int kRoleThreads = (kMmaWarp + 2) * 32, kLoadThreads = 64;
// Registers a thread: of the launch, and after the G warps have taken what the others do not need (whole warpgroups; an increase beyond
// what the block was launched with would wait for ever).
constexpr int kRegsLaunch = 96, kRegsG = 112, kRegsResult = 104, kRegsLoad = 48;
static_assert(kRegsG >= kRegsLaunch && kRegsResult >= kRegsLaunch && kRegsLoad <= kRegsLaunch, "inc, inc and dec below (the other direction is an illegal instruction)");
static_assert(kRegsLaunch * kRoleThreads <= 65536, "the launch's registers fit the multiprocessor");
static_assert(kFG * 128 * kRegsG + kRG * 128 * kRegsResult + 128 * kRegsLoad <= kRegsLaunch * kRoleThreads, "the roles' registers are the launch's");
constexpr int kRoleReserve = 6656;                           // static shared memory, kept out of the dynamic budget
constexpr int kMaxG = 4, kMaxP = 4, kUnscales = 16;
// Rows whose dictionary sums stay in tensor memory: its additions cut off, so every one shrinks the sum by a third of 2^-24 (8 rows, 64
// additions: 1.1e-6 too small; 4 rows: half of that). Segment m of the block is accumulated in buffer m & 1 and taken by that result group.
constexpr int kSegment = 4;
__device__ __forceinline__ int segments(int rows) { return (rows + kSegment - 1) / kSegment; }
// G tiles (those of 7 x 7 are twice as large). At least as many as groups: a group that waits for a tile's use u must know that use u - 2
// is over (a barrier tells only the parity of its phase); its own row before, kFG rows back, waited for the row kRing before that one.
template <int K> constexpr int kRing = K == 7 ? 2 : kMaxG;
static_assert(kRing<7> >= kFG && kRing<5> >= kFG, "a group is never two uses ahead of a ring entry");

struct __align__(16) RoleCtl {
    GradCtl c;                                               // (its mma / full barriers are not used)
    uint64_t g_full[kMaxG], g_empty[kMaxG], p_full[kMaxP], p_empty[kMaxP];
    uint64_t c_full[2], c_empty[2], d_full[2], d_empty[2];
    float unscale[kUnscales];                                // of the tiles, by number
    float back[128];                                         // 2^e of each plane's atom (0: a plane outside the subset)
    uint32_t listed[kRG][128][4];                            // lists: the pixels of a group's row that list the atom
};

struct RoleParams {
    GradTcParams b;
    int atoms;                   // rows of the first product: D, or s of a compact subset
    int d_block;                 // bytes of a column of them
    int planes_in, planes_out;   // of a frame in coef and gcoef
    int p_stages;
    int tma_in, tma_out;
    int out_pairs;               // results stored two pixels at a time (where not by TMA)
    int copy_bytes;              // coefficients by asynchronous copies of this size; 0 = TMA or one by one
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
    s.out = s.D + (p.want_coef ? GGeo<K>::BLOCKS * p.d_block : 0);
    s.Phi = s.out + (p.want_coef ? kRG * kOutBytes : 0);
    s.f = carve_floats(s.Phi + p.p_stages * p.b.stage_bytes, p.b, GGeo<K>::UW);
    return s;
}

__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile WaitCtx* wc, bool ok)
{
    return __all_sync(0xffffffffu, ok && mbar_wait(bar, parity, wc));
}

// ---- G warps ----------------------------------------------------------------------------------------------------------------

template <int K> __device__ __forceinline__ bool g_role(const RoleParams& p, RoleCtl& ctl, const RoleSmem<K>& s, int tid)
{
    using G = GGeo<K>;
    const int grp = __shfl_sync(0xffffffffu, tid >> 5, 0) / 4, x = tid % kGroupThreads, C = p.b.g.pb.c;
    volatile WaitCtx* wc = &ctl.c.wait;
    TileState<K, kFG, true> ts;
    Tiles tl(p.b.g);
    ts.start(p.b, tl, s.f, tid, grp);                            // (row `grp` is the group's first of the block)
    bool ok = true;
    int parity = 0;
    for (; tl.more(p.b.g); parity ^= 1) {
        const int base = tl.base, rows = tl.rows, n = tl.n;
        const bool inside = tl.x0 + x < p.b.g.pb.W;
        const int first = (grp + kFG - base % kFG) % kFG;                // the group's first row of the tile
        tl.next(p.b.g);                                                  // (the tile after it is asked for while this one is made)
        if (!(ok = ts.make(p.b, ctl.c, tl, parity, s.f, tid, ok, first, (grp + kFG - tl.base % kFG) % kFG, &ctl.unscale[n % kUnscales]))) break;
        for (int row = first; row < rows; row += kFG) {
            float v[G::kk];
            patch_grad<K>(s.f.U + row * G::UW + x, p.b.g.uh * G::UW, s.f.g + row * C * kGroupThreads + x, C, ts.scale, v, [] {});
            if (!inside) {
#pragma unroll
                for (int j = 0; j < G::kk; ++j) v[j] = 0.f;              // (patches of columns beyond the image may be anything)
            }
            const int item = base + row, st = item % kRing<K>;
            ok = wait_all(&ctl.g_empty[st], ((item / kRing<K>) & 1) ^ 1, wc, ok);
            if (ok) write_row<K>(s.G + st * G::G_BYTES, 128 * 128, x, v);
            fence_proxy_async_smem();
            mbar_arrive(&ctl.g_full[st]);
        }
    }
    cp_async_wait_all_();
    return ok;
}

__device__ __forceinline__ bool load_barrier_and(bool ok)
{
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 6, %2, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((int)ok), "n"(kLoadThreads) : "memory");
    return r != 0;
}

// ---- load warps ---------------------------------------------------------------------------------------------------------------

template <bool FAST> __device__ __forceinline__ void load_role(const CUtensorMap* map, const RoleParams& p, RoleCtl& ctl, uint8_t* sPhi, int tid)
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
                if (!(ok = mbar_wait(&ctl.p_empty[st], ((item / p.p_stages) & 1) ^ 1, wc))) break;
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
    if (FAST || p.copy_bytes) {
        // asynchronous copies of 16, 8 or 4 bytes (eight pixels to two): planes picked one by one, widths and addresses TMA does not take
        const int px = p.copy_bytes / 2, per = 128 / px, total = per * p.b.rows;
        const bool pick = p.b.mode == kModeGlobal && !(pb.flags & SR_COEF_COMPACT);
        bool go = true;
        for (Tiles tl(p.b.g); tl.more(p.b.g) && go; tl.next(p.b.g))
            for (int row = 0; row < tl.rows; ++row) {
                const int item = tl.base + row, st = item % p.p_stages;
                if (!(go = wait_all(&ctl.p_empty[st], ((item / p.p_stages) & 1) ^ 1, wc, go))) break;
                const uint32_t stage = smem_u32(sPhi + st * p.b.stage_bytes);
                const __half* src = p.b.coef + (int64_t)tl.f * p.planes_in * HW + (int64_t)(tl.y0 + row) * pb.W + tl.x0;
                for (int i = tid; i < total; i += kLoadThreads) {
                    const int l = i / per, x = (i - l * per) * px;       // (per is 16, 32 or 64)
                    const bool inside = tl.x0 + x < pb.W;
                    const uint32_t dst = stage + (x >> 6) * p.b.chunk_bytes + l * 128 + ((((x & 63) >> 3) ^ (l & 7)) << 4) + (x & 7) * 2;
                    const __half* from = src + (int64_t)(pick ? ctl.c.atoms[l] : l) * HW + (inside ? x : 0);
                    if (px == 8) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from), "r"(inside ? 16 : 0) : "memory");
                    else if (px == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(from), "r"(inside ? 8 : 0) : "memory");
                    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(from), "r"(inside ? 4 : 0) : "memory");
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&ctl.p_full[st])) : "memory");
            }
        cp_async_wait_all_();
        return;
    }
    const int s = pb.s;
    const bool lists = p.b.mode == kModeIdx || p.b.mode == kModeCompact;
    const bool gather = p.b.mode == kModeGlobal && !(pb.flags & SR_COEF_COMPACT);      // (odd widths)
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
                    for (int l0 = 0; l0 < p.b.rows; l0 += 16) {
                        __half h[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            h[i] = inside && l0 + i < p.b.rows ? __ldg(src + (int64_t)(gather ? ctl.c.atoms[l0 + i] : l0 + i) * HW) : zero;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
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

// One warp a product: the issue of one row's instructions takes a single warp some thousand cycles on a busy multiprocessor.
template <int K, bool COEF> __device__ __forceinline__ void mma_role(const RoleParams& p, RoleCtl& ctl, const RoleSmem<K>& s, uint32_t tmem)
{
    using G = GGeo<K>;
    volatile WaitCtx* wc = &ctl.c.wait;
    const uint64_t g_desc0 = COEF ? make_smem_desc(smem_u32(s.G), 16, 1024, kSwizzle128B)               // rows: K-major
                                  : make_smem_desc(smem_u32(s.G), 128 * 128, 1024, kSwizzle128B);       // columns: MN-major
    const uint64_t a_desc0 = make_smem_desc(smem_u32(COEF ? s.D : s.Phi), 16, 1024, kSwizzle128B);
    constexpr uint32_t kGLo = (G::BLOCKS == 2 ? 128 * 128 : G::LO_CHUNK * 16) >> 4;
    const uint32_t kDLo = (uint32_t)(G::BLOCKS == 2 ? p.d_block : G::LO_CHUNK * 16) >> 4, a_chunk = (uint32_t)p.b.chunk_bytes >> 4;
    constexpr uint32_t idesc = COEF ? make_idesc_f16(128, 128, false, false) : make_idesc_f16(128, G::NB, false, true);
    bool lose = p.b.lose != 0 && blockIdx.x == 0 && (COEF || !p.want_coef);
    bool ok = true;
    int gs = 0, ps = 0, seg = 0;                             // ring entries of the row; segment
    uint32_t gp = 0, pp = 0;                                 // and the parities of their uses
    for (Tiles tl(p.b.g); tl.more(p.b.g) && ok; tl.next(p.b.g)) {
        for (int row = 0; row < tl.rows; ++row) {
            const int item = tl.base + row;
            if (COEF) ok = wait_all(&ctl.c_empty[item & 1], ((item >> 1) & 1) ^ 1, wc, ok);
            else if (row % kSegment == 0) ok = wait_all(&ctl.d_empty[seg & 1], ((seg >> 1) & 1) ^ 1, wc, ok);
            if (!COEF) ok = wait_all(&ctl.p_full[ps], pp, wc, ok);
            ok = wait_all(&ctl.g_full[gs], gp, wc, ok);
            if (!ok) break;
            if (!COEF && p.copy_bytes) fence_proxy_async_smem();         // (written by cp.async, read by the tensor core)
            tc_fence_after_sync();
            if (elect_one()) {
                const uint64_t gd = g_desc0 + ((uint32_t)(gs * G::G_BYTES) >> 4);
                if (COEF) {
                    const uint32_t acc = tmem + (item & 1) * 128;
#pragma unroll
                    for (int ks = 0; ks < G::KSTEPS; ++ks) {
                        mma_f16_ss(acc, a_desc0 + 2 * ks, gd + 2 * ks, idesc, ks > 0);
                        mma_f16_ss(acc, a_desc0 + 2 * ks, gd + 2 * ks + kGLo, idesc, 1u);
                        mma_f16_ss(acc, a_desc0 + 2 * ks + kDLo, gd + 2 * ks, idesc, 1u);
                    }
                    if (!lose) mma_commit(&ctl.c_full[item & 1]);
                } else {
                    const uint32_t acc = tmem + 256 + (seg & 1) * G::NB;
                    const uint64_t ad = a_desc0 + ((uint32_t)(ps * p.b.stage_bytes) >> 4);
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        mma_f16_ss(acc, ad + (ks >> 2) * a_chunk + (ks & 3) * 2, gd + (uint32_t)(ks * 2048 >> 4), idesc, row % kSegment > 0 || ks > 0);
                    if (!lose) mma_commit(&ctl.p_empty[ps]);
                    if (row % kSegment == kSegment - 1 || row == tl.rows - 1) mma_commit(&ctl.d_full[seg & 1]);
                }
                mma_commit(&ctl.g_empty[gs]);
            }
            __syncwarp();
            lose = false;
            if (row % kSegment == kSegment - 1 || row == tl.rows - 1) ++seg;
            if (++gs == kRing<K>) { gs = 0; gp ^= 1; }
            if (++ps == p.p_stages) { ps = 0; pp ^= 1; }
        }
    }
    // tensor memory is freed only once every product has finished
    if (elect_one()) { mma_commit(&ctl.c.drain); mbar_wait_drain(&ctl.c.drain, 0); }
    __syncwarp();
}

// Two products with one factor, packed.
__device__ __forceinline__ void times2(float& x, float& y, float a, float b, float k)
{
    asm("{\n\t.reg .b64 v, f;\n\tmov.b64 v, {%2, %3};\n\tmov.b64 f, {%4, %4};\n\tmul.rn.f32x2 v, v, f;\n\tmov.b64 {%0, %1}, v;\n\t}"
        : "=f"(x), "=f"(y) : "f"(a), "f"(b), "f"(k));
}

// ---- result warps ---------------------------------------------------------------------------------------------------------------

template <int K, bool FAST> __device__ __forceinline__ void result_role(const CUtensorMap* map, const RoleParams& p, RoleCtl& ctl, const RoleSmem<K>& s, uint32_t tmem, int grp, int tid)
{
    using G = GGeo<K>;
    const Problem& pb = p.b.g.pb;
    volatile WaitCtx* wc = &ctl.c.wait;
    auto result_barrier = [&](bool go) { return group_barrier_and(2 + grp, go); };
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, l = 32 * warp + lane, W = pb.W;
    const int64_t HW = (int64_t)pb.H * W;
    const uint32_t at = tmem + ((uint32_t)(32 * warp) << 16), acc_at = at + grp * 128;
    constexpr int STEP = K == 7 ? 16 : 32;                   // accumulator columns at a time (registers)
    const bool listed = !FAST && p.b.mode == kModeIdx, compact = !FAST && p.b.mode == kModeCompact;
    const bool together = p.want_coef && (listed || compact);        // these meet at barriers, so they leave together
    const bool mine = 32 * warp < p.atoms;                   // this warp has atoms
    const float back = p.want_coef && l < p.atoms ? ctl.back[l] : 0.f;
    float total[G::kk];
#pragma unroll
    for (int j = 0; j < G::kk; ++j) total[j] = 0.f;
    uint8_t* chunk = s.out + grp * kOutBytes;                // 64 pixels of the group's 128 atoms
    uint8_t* to = chunk + warp * 4096;
    bool ok = true;
    int seg = 0;
    for (Tiles tl(p.b.g); tl.more(p.b.g) && ok; tl.next(p.b.g)) {
        for (int row = (tl.base + grp) & 1; p.want_coef && row < tl.rows; row += kRG) {      // rows whose number is grp modulo 2
            const int item = tl.base + row;
            const int64_t pix = (int64_t)(tl.y0 + row) * W + tl.x0;
            const uint32_t whole = back != 0.f ? ~0u : 0u;
            uint32_t keep[4] = {0u, 0u, 0u, 0u};
            if (listed) {                                    // which of the row's pixels list this lane's atom
                if (!(ok = result_barrier(ok))) break;       // the row before has been read
#pragma unroll
                for (int i = 0; i < 4; ++i) ctl.listed[grp][tid][i] = 0u;
                if (!(ok = result_barrier(ok))) break;
                if (tl.x0 + tid < W)
                    for (int q = 0; q < pb.s; ++q) {
                        const int a = min((int)__ldg(p.b.idx + ((int64_t)tl.f * pb.s + q) * HW + pix + tid), pb.D - 1);
                        atomicOr(&ctl.listed[grp][a][tid >> 5], 1u << (tid & 31));
                    }
            }
            ok = wait_all(&ctl.c_full[grp], (item >> 1) & 1, wc, ok);
            if (listed) {
                if (!(ok = result_barrier(ok))) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) keep[i] = ctl.listed[grp][l][i];
            }
            tc_fence_after_sync();
            const float k = back * *(volatile float*)&ctl.unscale[tl.n % kUnscales];
#pragma unroll
            for (int c0 = 0; c0 < 128; c0 += 64) {
                if (compact) {
                    if (!(ok = result_barrier(ok))) break;   // the chunk before has been taken
                }
#pragma unroll
                for (int c1 = 0; c1 < 64; c1 += STEP) {
                    float acc[STEP];
                    if (mine && ok) {
#pragma unroll
                        for (int i = 0; i < STEP; i += 16) tmem_ld_x16(acc_at + c0 + c1 + i, acc + i);
                    }
                    if (c1 == 0 && !compact) {
                        if (lane == 0) bulk_wait_read();     // the store before has read the buffer
                        __syncwarp();
                    }
                    if (mine && ok) {
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < STEP / 8; ++j) {
                            uint32_t h[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float a, b;
                                times2(a, b, acc[8 * j + 2 * i], acc[8 * j + 2 * i + 1], k);
                                const __half2 v2 = __floats2half2_rn(a, b);
                                h[i] = *reinterpret_cast<const uint32_t*>(&v2) & whole;      // (an atom outside the subset: zeros, whatever G is)
                            }
                            if (listed) {                    // pixels that do not list the atom
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const uint32_t two = keep[(c0 + c1 + 8 * j + 2 * i) / 32] >> ((c0 + c1 + 8 * j + 2 * i) % 32);
                                    h[i] &= ((two & 1u) ? 0xFFFFu : 0u) | ((two & 2u) ? 0xFFFF0000u : 0u);
                                }
                            }
                            *reinterpret_cast<uint4*>(to + lane * 128 + (((c1 / 8 + j) ^ (lane & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                        }
                    }
                }
                if (c0 == 64) {                              // the accumulator has been read
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.c_empty[grp]);
                }
                if (compact) {
                    // values by rank: a pixel's listed atoms out of the chunk
                    if (!(ok = result_barrier(ok))) break;
                    const int px = tid & 63;
                    if (tl.x0 + c0 + px < W)
                        for (int q = tid >> 6; q < pb.s; q += 2) {
                            const int64_t pl = ((int64_t)tl.f * pb.s + q) * HW + pix + c0 + px;
                            const int a = min((int)__ldg(p.b.idx + pl), pb.D - 1);
                            p.b.gcoef[pl] = *reinterpret_cast<const __half*>(chunk + (a >> 5) * 4096 + (a & 31) * 128 +
                                                                            ((((px >> 3) ^ (a & 7))) << 4) + (px & 7) * 2);
                        }
                } else if (FAST || p.tma_out) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0 && mine && ok && tl.x0 + c0 < W) {
                        tma_store_4d(map, to, tl.x0 + c0, tl.y0 + row, 32 * warp, tl.f);
                        bulk_commit();
                    }
                } else if (mine && ok) {
                    // any alignment: a plane's 64 pixels a warp, two elements a lane
                    __syncwarp();
                    __half* dst = p.b.gcoef + ((int64_t)tl.f * p.planes_out + 32 * warp) * HW + pix + c0;
                    const int left = W - tl.x0 - c0, most = min(32, p.atoms - 32 * warp);
                    if (p.out_pairs) {                       // (W even: a pair is inside or not)
                        if (2 * lane < left)
#pragma unroll 8
                            for (int a = 0; a < most; ++a)
                                *reinterpret_cast<uint32_t*>(dst + (int64_t)a * HW + 2 * lane) =
                                    *reinterpret_cast<const uint32_t*>(to + a * 128 + (((lane >> 2) ^ (a & 7)) << 4) + (lane & 3) * 4);
                    } else {
#pragma unroll 2
                        for (int half = 0; half < 64; half += 32) {
                            const int px = lane + half;
                            if (px < left)
#pragma unroll 8
                                for (int a = 0; a < most; ++a)
                                    dst[(int64_t)a * HW + px] = *reinterpret_cast<const __half*>(to + a * 128 + (((px >> 3) ^ (a & 7)) << 4) + (px & 7) * 2);
                        }
                    }
                    __syncwarp();
                }
            }
            if (!ok) break;
        }
        for (const int stop = seg + segments(tl.rows); seg < stop && p.want_dict && ok; ++seg) {
            if ((seg & 1) != grp) continue;
            ok = wait_all(&ctl.d_full[grp], (seg >> 1) & 1, wc, ok);
            if (together) ok = result_barrier(ok);
            tc_fence_after_sync();
            if (!ok) break;
            const float un = *(volatile float*)&ctl.unscale[tl.n % kUnscales];
            if (32 * warp < p.b.rows) {
                const uint32_t d = at + 256 + grp * G::NB;
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
            if (lane == 0) mbar_arrive(&ctl.d_empty[grp]);
        }
    }
    if (lane == 0) bulk_wait_all();
    // the groups' sums added in their order, through shared memory that every role has left by now
    tc_fence_before_sync();
    __syncthreads();                                         // (the block's last barrier: the other roles' is in the kernel)
    if (p.want_dict) {
        float* sum = reinterpret_cast<float*>(s.G);          // (49 x 128 floats at most, less than a ring)
        if (grp == 1 && l < p.b.rows) {
#pragma unroll
            for (int j = 0; j < G::kk; ++j) sum[j * 128 + l] = total[j];
        }
        asm volatile("barrier.cta.sync 4, %0;" ::"n"(kRG * kGroupThreads) : "memory");
        if (grp == 0 && l < p.b.rows) {
            float* out = p.b.partial + ((int64_t)blockIdx.x * p.b.rows + l) * G::kk;
#pragma unroll
            for (int j = 0; j < G::kk; ++j) out[j] = total[j] + sum[j * 128 + l];
        }
    }
}

// FAST: results by TMA, coefficients by TMA or asynchronous copies; without the other ways' code its roles keep their values in registers
// (1080p x4: 188 -> 172 us).
template <int K, bool FAST>
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

    init_ctl(ctl.c, p.b, tid, kRoleThreads, p.want_coef + p.want_dict);
    if (tid == 0) {
        for (int i = 0; i < kMaxG; ++i) { mbar_init(&ctl.g_full[i], kGroupThreads); mbar_init(&ctl.g_empty[i], p.want_coef + p.want_dict); }
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
        for (int q = tid; q < p.atoms; q += kRoleThreads) ctl.back[q] = write_atom<K>(p.b, s.D, p.d_block, q);
    fence_proxy_async_smem();
    if (warp == kMmaWarp) tmem_alloc(&ctl.c.tmem_base, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = ctl.c.tmem_base;

    // (setmaxnreg: whole warpgroups)
    if (warp < kResultWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsG));
        g_role<K>(p, ctl, s, tid);
    } else if (warp < kLoadWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsResult));
        result_role<K, FAST>(&map_out, p, ctl, s, tmem, (warp - kResultWarp) / 4, (tid - kResultWarp * 32) % kGroupThreads);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLoad));
        if (warp == kMmaWarp) { if (p.want_coef) mma_role<K, true>(p, ctl, s, tmem); }
        else if (warp == kMmaWarp + 1) { if (p.want_dict) mma_role<K, false>(p, ctl, s, tmem); }
        else if (p.want_dict) load_role<FAST>(&map_in, p, ctl, s.Phi, tid - kLoadWarp * 32);
    }

    if (warp < kResultWarp || warp >= kLoadWarp) {
        __syncwarp();
        tc_fence_before_sync();
        __syncthreads();                                     // (the result warps': in their role)
        tc_fence_after_sync();
    }
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
    p.d_block = ((p.atoms + 7) & ~7) * 128;              // (the product reads 128 rows; those behind are whatever follows)
    p.b.rows = grad_rows(a);
    p.b.stage_bytes = stage_bytes_of(p.b.rows);
    p.b.chunk_bytes = p.b.stage_bytes / 2;
    const size_t floats = float_bytes<K>(p.b.g, a.pb, a.lr);
    // (behind the atoms lie 16 KB and more of results, so what the first product reads there is shared memory)
    const size_t fixed = 1024 + (size_t)kRing<K> * GGeo<K>::G_BYTES + (p.want_coef ? GGeo<K>::BLOCKS * p.d_block + kRG * kOutBytes : 0) + floats;
    p.p_stages = 0;
    smem = fixed;
    if (p.want_dict) {
        for (p.p_stages = kMaxP; p.p_stages >= 2; --p.p_stages) {
            smem = fixed + (size_t)p.p_stages * p.b.stage_bytes;
            // the second product reads 128 rows of a chunk, whatever lies behind the last one must be shared memory
            const size_t reach = smem - floats - p.b.chunk_bytes + 128 * 128;
            if (smem < reach) smem = reach;
            if (fits(smem, kRoleReserve)) break;
        }
        if (p.p_stages < 2) return false;
    }
    return fits(smem, kRoleReserve);
}

template <int K, bool FAST> cudaError_t launch_form(const CUtensorMap& in, const CUtensorMap& out, const RoleParams& p, int blocks, size_t smem, cudaStream_t st)
{
    static bool done[64] = {false};
    if (cudaError_t e = allow_smem(grad_roles_kernel<K, FAST>, done, kRoleReserve)) return e;
    grad_roles_kernel<K, FAST><<<blocks, kRoleThreads, smem, st>>>(in, out, p);
    count_launches(1);
    return cudaGetLastError();
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
    if (p.want_dict && !p.tma_in && (whole || a.mode == kModeGlobal))
        for (int bytes = 16; bytes >= 4 && !p.copy_bytes; bytes /= 2)
            if (pb.W % (bytes / 2) == 0 && ((uintptr_t)a.coef & (bytes - 1)) == 0) p.copy_bytes = bytes;
    if (p.want_coef && a.mode != kModeCompact && pb.W % 8 == 0 && ((uintptr_t)a.gcoef & 15) == 0) p.tma_out = encode_planes(&out, a.gcoef, pb, p.planes_out, 32);
    p.out_pairs = pb.W % 2 == 0 && ((uintptr_t)a.gcoef & 3) == 0;
    const bool fast = (!p.want_coef || p.tma_out) && (!p.want_dict || p.tma_in || p.copy_bytes) && a.mode != kModeIdx;
    *slots = p.b.g.num_tiles < sm_count() ? p.b.g.num_tiles : sm_count();
    return fast ? launch_form<K, true>(in, out, p, *slots, smem, a.st) : launch_form<K, false>(in, out, p, *slots, smem, a.st);
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
    // Two load warps without asynchronous copies do not keep up with whole planes (odd widths: 1077 x 1080, D = 72: both gradients 686 us,
    // 537 by the two kernels of sr_grad_tc.cu), nor with the dictionary's sums over lists alone (1080p x4, s = 8: 473 / 303; both
    // gradients 545 / 768).
    const bool sums = a.gdict || a.ggamma;
    if (sums && (a.mode == kModeDense || a.mode == kModeGlobal) && (a.pb.W % 2 != 0 || ((uintptr_t)a.coef & 3) != 0)) return false;
    if (sums && !a.gcoef && (a.mode == kModeIdx || a.mode == kModeCompact)) return false;
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
