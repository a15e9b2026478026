// Both gradients of the dictionary regression in one kernel of specialised warps, for binary16 coefficients with at most 128 atoms:
// k in {3, 5, 7}, up to four channels, any width and every mode. (sr_grad_tc.cu: the mathematics, and more atoms.)
//
// What bounds a kernel whose warps do everything in turn is not the tensor core or memory but the waits between the steps of a row
// (1080p x4, D = 72, k = 5: 129 + 129 us in two kernels, 34 of each the up-sampled tile, against 95 us of traffic). Here one block per
// multiprocessor holds a pipeline, and G, which costs most, is computed once for both products:
//   G warps (kFG groups of four)   the up-sampled tile; G of every row, hi + lo, into a ring of tiles         g_full
//   load warps (two or six)         the row's coefficients into a ring of stages: TMA boxes (lists: masked      p_full
//                                  there), or (widths and addresses TMA does not take, gathered planes,
//                                  compact values) smaller asynchronous copies or a pixel a thread
//   MMA warps (one a product)      a row's coefficient gradients in one of two accumulators (lane = atom,     c_full, g_empty
//                                  column = pixel), the dictionary's sums over four rows in one of two more    d_full, p_empty, g_empty
//   result warps (kRG groups of four)  a row's coefficient gradients to memory (c_empty), those dictionary sums to registers (d_empty)
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
// What a kernel is compiled for. kFast: results by TMA, coefficients by TMA or asynchronous copies; without the other ways' code its roles
// keep their values in registers (1080p x4: 188 -> 162 us). kLists: lists, both by TMA. kGeneral: the rest. kPairs: the same with
// more load warps and fewer registers a warp.
enum Form { kGeneral, kPairs, kFast, kLists };
constexpr bool has_pairs(Form f) { return f == kPairs || f == kLists; }
constexpr int kResultWarp = kFG * 4, kLoadWarp = kResultWarp + kRG * 4, kLoadThreads = 64;
constexpr int kLoadPairs = 3;                                // pairs of load warps where there are more than one: a row a pair, in turn
template <Form F> constexpr int kMmaWarp = kLoadWarp + (has_pairs(F) ? 2 * kLoadPairs : 2);
template <Form F> constexpr int kRoleThreads = (kMmaWarp<F> + 2) * 32;
// Registers a thread: of the launch, and after the G warps have taken what the others do not need (whole warpgroups; an increase beyond
// what the block was launched with would wait for ever).
template <Form F> constexpr int kRegsLaunch = has_pairs(F) ? 80 : 96;
template <Form F> constexpr int kRegsG = has_pairs(F) ? 104 : 112;
template <Form F> constexpr int kRegsResult = has_pairs(F) ? 88 : 104;
constexpr int kRegsLoad = 48;
template <Form F> constexpr bool kRegsFit =
    kRegsG<F> >= kRegsLaunch<F> && kRegsResult<F> >= kRegsLaunch<F> && kRegsLoad <= kRegsLaunch<F> &&   // inc, inc, dec: the other direction is illegal
    kRoleThreads<F> % 128 == 0 && kRegsLaunch<F> * kRoleThreads<F> <= 65536 &&
    128 * (kFG * kRegsG<F> + kRG * kRegsResult<F> + (kRoleThreads<F> / 128 - kFG - kRG) * kRegsLoad) <= kRegsLaunch<F> * kRoleThreads<F>;
static_assert(kRegsFit<kGeneral> && kRegsFit<kPairs> && kRegsFit<kFast> && kRegsFit<kLists>, "the roles' registers are the launch's");
constexpr int kRoleReserve = 6656;                           // static shared memory, kept out of the dynamic budget
constexpr int kMaxG = 4, kMaxP = 4, kUnscales = 16;
// Rows whose dictionary sums stay in tensor memory: its additions cut off, so every one shrinks the sum by a third of 2^-24 (8 rows, 64
// additions: 1.1e-6 too small; 4 rows: half of that). Segment m of the block is accumulated in buffer m & 1 and taken by that result group.
constexpr int kSegment = 4;
__device__ __forceinline__ int segments(int rows) { return (rows + kSegment - 1) / kSegment; }
// G tiles (those of 7 x 7 are twice as large). At least as many as groups: a group that waits for a tile's use u must know that use u - 2
// is over (a barrier tells only the parity of its phase); its own row before, kFG rows back, waited for the row kRing before that one.
template <int K> constexpr int kRing = K == 7 ? 2 : kMaxG;
// Lists: rows of bits, one for each of a row's pixels and 128 atoms. Every stage has one pair of load warps, and every entry of bits one pair
// and one result group (two entries a pair), for the same reason: a wait for the use before follows that warp's own use before.
constexpr int kBitsRing = 2 * kLoadPairs, kBitsBytes = 128 * 16;
static_assert(kRG == 2, "two entries a pair");
static_assert(kRing<7> >= kFG && kRing<5> >= kFG, "a group is never two uses ahead of a ring entry");

struct __align__(16) RoleCtl {
    GradCtl c;
    uint64_t g_full[kMaxG], g_empty[kMaxG], p_full[kMaxP], p_empty[kMaxP];
    uint64_t c_full[2], c_empty[2], d_full[2], d_empty[2];
    uint64_t p_land[kMaxP], b_full[kBitsRing], b_empty[kBitsRing];
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
    int lists;                   // lists over planes that TMA takes: the load warps mask them, and make the bits for the result warps
    int pairs;                   // of load warps at work; if more than one, as many as stages
};

template <int K> struct RoleSmem {
    uint8_t *G, *D, *out, *bits, *Phi;
    Floats f;
};
// [G ring][atoms][results][bits][coefficient ring][floats]
template <int K> __device__ __forceinline__ RoleSmem<K> carve(uint8_t* at, const RoleParams& p)
{
    RoleSmem<K> s;
    s.G = at;
    s.D = s.G + kRing<K> * GGeo<K>::G_BYTES;
    s.out = s.D + (p.want_coef ? GGeo<K>::BLOCKS * p.d_block : 0);
    s.bits = s.out + (p.want_coef ? kRG * kOutBytes : 0);
    s.Phi = s.bits + (p.lists ? kBitsRing * kBitsBytes : 0);
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

__device__ __forceinline__ bool load_barrier_and(int pair, bool ok)
{
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %3, %2, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((int)ok), "n"(kLoadThreads), "r"(6 + pair) : "memory");
    return r != 0;
}

// ---- load warps ---------------------------------------------------------------------------------------------------------------

// A word of bits covers 32 pixels; pixel 4 t + i stands at bit 8 i + 7 - t, so that a shift by t brings four neighbours to the signs of the
// four bytes, and a permutation spreads those over 16-bit masks.
__device__ __forceinline__ int bit_of_pixel(int px) { return 8 * (px & 3) + 7 - (px >> 2); }
__device__ __forceinline__ void mask_four(uint32_t bits, int t, uint32_t& m01, uint32_t& m23)
{
    const uint32_t signs = bits << t;
    asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(m01) : "r"(signs));
    asm("prmt.b32 %0, %1, 0, 0xBBAA;" : "=r"(m23) : "r"(signs));
}

// Lists over whole planes: a row's planes land by TMA like those of the dense form, a warp takes 64 of its pixels, sets a bit for every
// (atom, pixel) that a list names, and clears the values without one in place; the result warps read the same bits. All planes are read for
// a few of each pixel's, but gathering those, two bytes at a time, waits for memory twice a row (1080p x4, D = 72, k = 5, s = 8: both
// gradients 554 us, coefficients 287, dictionary 306; so 247, 144, 162). The instructions of a row's bits and masks are too many for one
// pair of warps (335, 199, 286): three take a row each in turn. (Four planes' loads before their first store: 300, 147, 212.)
__device__ __forceinline__ void load_lists(const CUtensorMap* map, const RoleParams& p, RoleCtl& ctl, uint8_t* sPhi, uint8_t* sBits, int tid)
{
    const Problem& pb = p.b.g.pb;
    volatile WaitCtx* wc = &ctl.c.wait;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0) & 1, lane = tid & 31, s = pb.s;
    const int64_t HW = (int64_t)pb.H * pb.W;
    bool ok = true;
    int issued = -1;                                         // the last row asked for (in the pair's stage: the ones before have landed)
    auto issue = [&](int x0, int y, int f, int item) {
        if (warp != 0 || !p.want_dict) return;
        const int st = item % p.p_stages;
        ok = wait_all(&ctl.p_empty[st], ((item / p.p_stages) & 1) ^ 1, wc, ok);
        if (!ok) return;
        if (elect_one()) {
            uint8_t* dst = sPhi + st * p.b.stage_bytes;
            mbar_arrive_expect_tx(&ctl.p_land[st], (uint32_t)p.b.rows * 256u);
            tma_load_4d(dst, map, &ctl.p_land[st], x0, y, 0, f);
            tma_load_4d(dst + p.b.chunk_bytes, map, &ctl.p_land[st], x0 + 64, y, 0, f);
        }
        __syncwarp();
        issued = item;
    };
    // Sixteen ranks of the row: a lane takes four pixels of every other one (idx on four bytes, W % 8 == 0: all four inside or none).
    const int px = 4 * (lane & 15), odd = lane >> 4;
    uint32_t a[8];
    auto ask = [&](int x0, int y, int f, int q0) {
        const int x = x0 + 64 * warp + px;
        const uint8_t* at = p.b.idx + ((int64_t)f * s + q0 + odd) * HW + (int64_t)y * pb.W + x;
#pragma unroll
        for (int i = 0; i < 8; ++i, at += 2 * HW) a[i] = q0 + 2 * i + odd < s && x < pb.W ? __ldg(reinterpret_cast<const uint32_t*>(at)) : 0u;
    };
    // rows pair, pair + pairs, ... of the block's
    const int ring = 2 * p.pairs;
    Tiles tl(p.b.g);
    int row = tid / kLoadThreads, x0, y, f, item;
    if (row >= p.pairs) return;
    auto settle = [&]() { while (tl.more(p.b.g) && row >= tl.rows) { row -= tl.rows; tl.next(p.b.g); } };
    auto take = [&]() { x0 = tl.x0; y = tl.y0 + row; f = tl.f; item = tl.base + row; };
    settle();
    take();
    if (tl.more(p.b.g)) {
        issue(x0, y, f, item);
        ask(x0, y, f, 0);
    }
    while (tl.more(p.b.g) && ok) {
        const int bst = item % ring;
        if (p.want_coef) ok = wait_all(&ctl.b_empty[bst], ((item / ring) & 1) ^ 1, wc, ok);
        if (!ok) break;
        uint32_t* bits = reinterpret_cast<uint32_t*>(sBits + bst * kBitsBytes) + warp * 256;     // of the warp's pixels: [32 pixels][atom]
#pragma unroll
        for (int i = 0; i < 2; ++i) reinterpret_cast<uint4*>(bits)[lane + 32 * i] = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
        uint32_t* word = bits + (px >> 5) * 128;
        const uint32_t first = x0 + 64 * warp + px < pb.W ? 1u << bit_of_pixel(px & 31) : 0u;            // (px is the first of four: the others' are 8, 16, 24 higher)
        for (int q0 = 0;; ) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (q0 + 2 * i < s) {
                    const uint32_t bit = q0 + 2 * i + odd < s ? first : 0u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) atomicOr(word + min((int)(a[i] >> (8 * j) & 255u), pb.D - 1), bit << (8 * j));
                }
            if ((q0 += 16) >= s) break;
            ask(x0, y, f, q0);
        }
        const int at_row = item;
        row += p.pairs;
        settle();
        take();
        if (tl.more(p.b.g)) ask(x0, y, f, 0);
        __syncwarp();
        if (p.want_coef) mbar_arrive(&ctl.b_full[bst]);
        if (!p.want_dict) continue;
        const int st = at_row % p.p_stages;
        if (!(ok = wait_all(&ctl.p_land[st], (at_row / p.p_stages) & 1, wc, ok))) break;
        uint8_t* chunk = sPhi + st * p.b.stage_bytes + warp * p.b.chunk_bytes;
        const int unit = lane & 7;
#pragma unroll 4
        for (int l = lane >> 3; l < pb.D; l += 4) {
            const uint32_t b = bits[(unit >> 2) * 128 + l];
            uint4* at = reinterpret_cast<uint4*>(chunk + l * 128 + ((unit ^ (l & 7)) << 4));
            uint4 v = *at;
            uint32_t m0, m1, m2, m3;
            mask_four(b, 2 * (unit & 3), m0, m1);
            mask_four(b, 2 * (unit & 3) + 1, m2, m3);
            *at = make_uint4(v.x & m0, v.y & m1, v.z & m2, v.w & m3);
        }
        fence_proxy_async_smem();
        mbar_arrive(&ctl.p_full[st]);
        if (tl.more(p.b.g)) issue(x0, y, f, item);
    }
    // what was asked for lands before shared memory is given up
    if (!ok && issued >= 0) mbar_wait_drain(&ctl.p_land[issued % p.p_stages], (issued / p.p_stages) & 1);
}

template <Form FORM> __device__ __forceinline__ void load_role(const CUtensorMap* map, const RoleParams& p, RoleCtl& ctl, uint8_t* sPhi, int tid)
{
    const Problem& pb = p.b.g.pb;
    volatile WaitCtx* wc = &ctl.c.wait;
    const int64_t HW = (int64_t)pb.H * pb.W;
    const int pair = FORM == kPairs ? __shfl_sync(0xffffffffu, tid >> 6, 0) : 0;
    if (pair >= p.pairs) return;
    tid &= kLoadThreads - 1;
    if (FORM != kPairs && p.tma_in) {
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
    if (FORM == kFast || (FORM != kPairs && p.copy_bytes)) {
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
    if constexpr (FORM == kPairs) {                          // (whatever else asks for sums has returned: plan_best)
        const int s = pb.s;
        const bool lists = p.b.mode == kModeIdx || p.b.mode == kModeCompact;
        const bool gather = p.b.mode == kModeGlobal && !(pb.flags & SR_COEF_COMPACT);      // (odd widths)
        const __half zero = __ushort_as_half(0);
        bool ok = true;
        Tiles tl(p.b.g);
        for (int row = pair; tl.more(p.b.g); row += p.pairs) {
            while (tl.more(p.b.g) && row >= tl.rows) { row -= tl.rows; tl.next(p.b.g); }
            if (!tl.more(p.b.g)) break;
            const int item = tl.base + row, st = item % p.p_stages;
            uint8_t* stage = sPhi + st * p.b.stage_bytes;
            ok = wait_all(&ctl.p_empty[st], ((item / p.p_stages) & 1) ^ 1, wc, ok);
            if (lists) {
                if (ok)
                    for (int i = tid; i < p.b.stage_bytes / 16; i += kLoadThreads) reinterpret_cast<uint4*>(stage)[i] = make_uint4(0, 0, 0, 0);
                ok = load_barrier_and(pair, ok);                         // (a pair leaves together: its warps meet here)
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

template <int K, Form FORM> __device__ __forceinline__ void result_role(const CUtensorMap* map, const RoleParams& p, RoleCtl& ctl, const RoleSmem<K>& s, uint32_t tmem, int grp, int tid)
{
    using G = GGeo<K>;
    const Problem& pb = p.b.g.pb;
    volatile WaitCtx* wc = &ctl.c.wait;
    auto result_barrier = [&](bool go) { return group_barrier_and(2 + grp, go); };
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, l = 32 * warp + lane, W = pb.W;
    const int64_t HW = (int64_t)pb.H * W;
    const uint32_t at = tmem + ((uint32_t)(32 * warp) << 16), acc_at = at + grp * 128;
    constexpr int STEP = K == 7 ? 16 : 32;                   // accumulator columns at a time (registers)
    constexpr int kUnroll = FORM == kLists ? 1 : 2;          // (lists: less code for more roles; coefficients of lists 170 -> 144 us with the shorter masks)
    constexpr bool any = FORM == kGeneral || FORM == kPairs;
    const bool listed = any && p.b.mode == kModeIdx, compact = any && p.b.mode == kModeCompact;
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
                        atomicOr(&ctl.listed[grp][a][tid >> 5], 1u << bit_of_pixel(tid & 31));
                    }
            }
            if (FORM == kLists) {
                const int ring = 2 * p.pairs, bst = item % ring;
                ok = wait_all(&ctl.b_full[bst], (item / ring) & 1, wc, ok);
#pragma unroll
                for (int i = 0; i < 4; ++i) keep[i] = reinterpret_cast<const uint32_t*>(s.bits + bst * kBitsBytes)[i * 128 + l];
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.b_empty[bst]);
            }
            ok = wait_all(&ctl.c_full[grp], (item >> 1) & 1, wc, ok);
            if (listed) {
                if (!(ok = result_barrier(ok))) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) keep[i] = ctl.listed[grp][l][i];
            }
            tc_fence_after_sync();
            const float k = back * *(volatile float*)&ctl.unscale[tl.n % kUnscales];
#pragma unroll kUnroll
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
                            if (listed || FORM == kLists) {  // pixels that do not list the atom
                                const uint32_t b = (c1 + 8 * j) / 32 ? (c0 ? keep[3] : keep[1]) : (c0 ? keep[2] : keep[0]);
                                uint32_t m[4];
                                mask_four(b, (c1 + 8 * j) % 32 / 4, m[0], m[1]);
                                mask_four(b, (c1 + 8 * j) % 32 / 4 + 1, m[2], m[3]);
#pragma unroll
                                for (int i = 0; i < 4; ++i) h[i] &= m[i];
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
                } else if (!any || p.tma_out) {
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

template <int K, Form FORM>
__global__ void __launch_bounds__(kRoleThreads<FORM>, 1)
grad_roles_kernel(const __grid_constant__ CUtensorMap map_in, const __grid_constant__ CUtensorMap map_out, const __grid_constant__ RoleParams p)
{
    using G = GGeo<K>;
    constexpr int kThreads = kRoleThreads<FORM>, kMma = kMmaWarp<FORM>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ RoleCtl ctl;
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const RoleSmem<K> s = carve<K>(smem, p);
    const Problem& pb = p.b.g.pb;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), D = pb.D;

    init_ctl(ctl.c, p.b, tid, kThreads, p.want_coef + p.want_dict);
    if (tid == 0) {
        for (int i = 0; i < kMaxG; ++i) { mbar_init(&ctl.g_full[i], kGroupThreads); mbar_init(&ctl.g_empty[i], p.want_coef + p.want_dict); }
        for (int i = 0; i < kMaxP; ++i) { mbar_init(&ctl.p_full[i], p.tma_in && FORM != kLists ? 1 : kLoadThreads); mbar_init(&ctl.p_empty[i], 1); mbar_init(&ctl.p_land[i], 1); }
        for (int i = 0; i < kBitsRing; ++i) { mbar_init(&ctl.b_full[i], kLoadThreads); mbar_init(&ctl.b_empty[i], 4); }
        for (int i = 0; i < 2; ++i) { mbar_init(&ctl.c_full[i], 1); mbar_init(&ctl.c_empty[i], 4); mbar_init(&ctl.d_full[i], 1); mbar_init(&ctl.d_empty[i], 4); }
        fence_barrier_init();
        if (p.tma_in) prefetch_tensormap(&map_in);
        if (p.tma_out) prefetch_tensormap(&map_out);
    }
    // (what the products read beyond the atoms, planes and taps written ends in lanes and columns that nobody reads)
    for (int i = tid; i < pb.c * p.b.g.trows * p.b.g.tcols + 8; i += kThreads) s.f.L[i] = 0.f;
    if (p.b.mode == kModeGlobal && tid < pb.s) ctl.c.atoms[tid] = (uint8_t)min((int)__ldg(p.b.idx + tid), D - 1);
    __syncthreads();
    if (p.want_coef)
        for (int q = tid; q < p.atoms; q += kThreads) ctl.back[q] = write_atom<K>(p.b, s.D, p.d_block, q);
    fence_proxy_async_smem();
    if (warp == kMma) tmem_alloc(&ctl.c.tmem_base, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = ctl.c.tmem_base;

    // (setmaxnreg: whole warpgroups)
    if (warp < kResultWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsG<FORM>));
        g_role<K>(p, ctl, s, tid);
    } else if (warp < kLoadWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsResult<FORM>));
        result_role<K, FORM>(&map_out, p, ctl, s, tmem, (warp - kResultWarp) / 4, (tid - kResultWarp * 32) % kGroupThreads);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLoad));
        if (warp == kMma) { if (p.want_coef) mma_role<K, true>(p, ctl, s, tmem); }
        else if (warp == kMma + 1) { if (p.want_dict) mma_role<K, false>(p, ctl, s, tmem); }
        else if (FORM == kLists) load_lists(&map_in, p, ctl, s.Phi, s.bits, tid - kLoadWarp * 32);
        else if (p.want_dict) load_role<FORM>(&map_in, p, ctl, s.Phi, tid - kLoadWarp * 32);
    }

    if (warp < kResultWarp || warp >= kLoadWarp) {
        __syncwarp();
        tc_fence_before_sync();
        __syncthreads();                                     // (the result warps': in their role)
        tc_fence_after_sync();
    }
    if (ctl.c.wait.abort_flag && tid == 0) atomicExch(p.b.status, SR_ERR_TIMEOUT);
    if (warp == kMma) tmem_dealloc(tmem, 512);
}

// ---- host ------------------------------------------------------------------------------------------------------------------------

int out_planes(const GradArgs& a) { return a.mode == kModeCompact || (a.mode == kModeGlobal && (a.pb.flags & SR_COEF_COMPACT)) ? a.pb.s : a.pb.D; }
int product_atoms(const GradArgs& a) { return a.mode == kModeGlobal && (a.pb.flags & SR_COEF_COMPACT) ? a.pb.s : a.pb.D; }

bool tma_takes(const Problem& pb, const void* at) { return pb.W % 8 == 0 && ((uintptr_t)at & 15) == 0; }

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
    const size_t fixed = 1024 + (size_t)kRing<K> * GGeo<K>::G_BYTES + (p.want_coef ? GGeo<K>::BLOCKS * p.d_block + kRG * kOutBytes : 0) +
                         (p.lists ? kBitsRing * kBitsBytes : 0) + floats;
    p.p_stages = 0;
    smem = fixed;
    if (p.want_dict) {
        for (p.p_stages = p.pairs > 1 ? kLoadPairs : kMaxP; p.p_stages >= 2; --p.p_stages) {
            smem = fixed + (size_t)p.p_stages * p.b.stage_bytes;
            // the second product reads 128 rows of a chunk, whatever lies behind the last one must be shared memory
            const size_t reach = smem - floats - p.b.chunk_bytes + 128 * 128;
            if (smem < reach) smem = reach;
            if (fits(smem, kRoleReserve)) break;
        }
        if (p.p_stages < 2) return false;
        if (p.pairs > 1) p.pairs = p.p_stages;
    }
    return fits(smem, kRoleReserve);
}

// Bytes of an asynchronous copy that W and the address of the planes take, or 0.
int copy_of(const Problem& pb, const void* at)
{
    for (int bytes = 16; bytes >= 4; bytes /= 2)
        if (pb.W % (bytes / 2) == 0 && ((uintptr_t)at & (bytes - 1)) == 0) return bytes;
    return 0;
}

// Whole planes that lanes load pixel by pixel (odd widths): from how many on three pairs of load warps beat the two kernels of
// sr_grad_tc.cu, whose every warp loads. Both gradients, 1080 rows of 1077 pixels, scale 3, us, two kernels / pairs, k = 5: D = 32
// 278 / 316, 40 333 / 349, 56 404 / 369, 72 680 / 428. The number is k = 5's. At k = 7 the pairs win from 16 planes on (16 448 / 292, 40
// 714 / 420, 72 988 / 491), at k = 3 the two kernels up to 72 (40 251 / 305, 72 354 / 377), on small frames up to 40 (3 x 255 x 271:
// 40 85 / 93, 72 138 / 107). Compact values and lists, 1080p x4, D = 72, s = 8, one pair / three: compact 423 / 310, its
// dictionary sums alone 202 (two kernels' form) / 181; at k = 7 507 / 355, 699 / 265.
constexpr int kPairsPlanes = 40;
bool one_by_one(const GradArgs& a) { return (a.gdict || a.ggamma) && a.mode != kModeIdx && a.mode != kModeCompact && copy_of(a.pb, a.coef) == 0; }

// With lists masked in place where that fits and TMA takes the planes.
template <int K> bool plan_best(RoleParams& p, const GradArgs& a, size_t& smem)
{
    const bool sums = a.gdict || a.ggamma;
    p.pairs = kLoadPairs;
    p.lists = a.mode == kModeIdx && ((uintptr_t)a.idx & 3) == 0 && (!sums || tma_takes(a.pb, a.coef)) && (!a.gcoef || tma_takes(a.pb, a.gcoef));
    if (p.lists && plan<K>(p, a, smem)) return true;
    p.lists = 0;
    p.pairs = sums && (a.mode == kModeIdx || a.mode == kModeCompact || one_by_one(a)) ? kLoadPairs : 1;
    return plan<K>(p, a, smem);
}

template <int K, Form FORM> cudaError_t launch_form(const CUtensorMap& in, const CUtensorMap& out, const RoleParams& p, int blocks, size_t smem, cudaStream_t st)
{
    static bool done[64] = {false};
    if (cudaError_t e = allow_smem(grad_roles_kernel<K, FORM>, done, kRoleReserve)) return e;
    grad_roles_kernel<K, FORM><<<blocks, kRoleThreads<FORM>, smem, st>>>(in, out, p);
    count_launches(1);
    return cudaGetLastError();
}

template <int K> cudaError_t launch_k(const GradArgs& a, int* slots)
{
    RoleParams p{};
    p.b = common_params(a);
    if (!p.b.status) return cudaErrorUnknown;
    size_t smem = 0;
    if (!plan_best<K>(p, a, smem)) return cudaErrorNotSupported;
    p.planes_out = out_planes(a);
    p.planes_in = p.planes_out;
    CUtensorMap in{}, out{};
    const Problem& pb = a.pb;
    const bool whole = a.mode == kModeDense || (a.mode == kModeGlobal && (pb.flags & SR_COEF_COMPACT));
    if (p.want_dict && (whole || p.lists) && tma_takes(pb, a.coef)) p.tma_in = encode_planes(&in, a.coef, pb, p.planes_in, p.b.rows);
    if (p.want_dict && !p.tma_in && (whole || a.mode == kModeGlobal))
        p.copy_bytes = copy_of(pb, a.coef);
    if (p.want_coef && a.mode != kModeCompact && tma_takes(pb, a.gcoef)) p.tma_out = encode_planes(&out, a.gcoef, pb, p.planes_out, 32);
    p.out_pairs = pb.W % 2 == 0 && ((uintptr_t)a.gcoef & 3) == 0;
    const bool ways = (!p.want_coef || p.tma_out) && (!p.want_dict || p.tma_in || p.copy_bytes);
    if (p.lists && !ways) return cudaErrorUnknown;           // (no encoder of tensor maps)
    *slots = p.b.g.num_tiles < sm_count() ? p.b.g.num_tiles : sm_count();
    if (p.lists) return launch_form<K, kLists>(in, out, p, *slots, smem, a.st);
    if (p.pairs > 1) return launch_form<K, kPairs>(in, out, p, *slots, smem, a.st);
    return ways && a.mode != kModeIdx ? launch_form<K, kFast>(in, out, p, *slots, smem, a.st) : launch_form<K, kGeneral>(in, out, p, *slots, smem, a.st);
}

template <int K> bool plan_fits(const GradArgs& a)
{
    RoleParams p{};
    size_t smem;
    return plan_best<K>(p, a, smem);
}

} // namespace

bool grad_roles_supported(const GradArgs& a)
{
    if (!form_supported(a) || a.pb.D > 128) return false;
    if (one_by_one(a) && grad_rows(a) < kPairsPlanes) return false;
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
