"""Gradients of the regression (dense, per-pixel lists, compact values, global subset) against the fp64 definition, against
differences of the oracle's forward pass, and the calls around them: parts that are not asked for, streams, graphs, misaligned and
offset tensors, values that are not finite.

Bounds. A gradient of a coefficient is a sum of k*k products of an atom's tap with G, itself c products of grad_out with an up-sampled
value of 4 + 4 weighted taps; sum_terms |.| (second value of `train_ref.grads`) is the sum of its terms' magnitudes with every LR tap's.
A chain of N fp32 operations is off by at most N half-steps of that sum. N = k*k + c + 16 in fp32 arithmetic; the tensor cores hold G and the
atoms as two binary16 numbers each (22 bits: 2^-22 = 4 half-steps per factor, and the product of the two low parts, 4 more, is left
out) and cut each of their sums' additions off instead of rounding it (two half-steps each). So 2 (k*k + c + 16) + 16 covers both. A
binary16 result adds its own half step, and half of 2^-24 among the subnormals. A gradient of the dictionary is a chain over the
pixels of a tile (at most 128 in fp32; 1024 in steps of 16 on the tensor cores: 64 additions cut off) and then over a block's tiles.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2303_08999_b200 as sr
import sr_inputs
import train_ref
from gpu_util import host, signed_asymmetric_dictionary, signed_gamma
from train_ref import U16, U32, to

pytestmark = pytest.mark.gpu


def _inputs(n, c, h, w, r, D, k, dt, seed=1):
    wl = sr_inputs.Workload("t", n, c, h, w, r, D=D, k=k, coef_dtype=dt)
    lr, d, coef = sr_inputs.make_inputs(wl, seed=sr_inputs.BASE_SEED + seed)
    d = signed_asymmetric_dictionary(d, seed=seed)
    d = np.where(np.isfinite(d), d, np.float32(0.5))         # a difference of Gaussians of one tap divided by its sum is 0 / 0
    gout = np.random.default_rng(seed).normal(0.0, 0.05, (n, c, h * r, w * r)).astype(np.float32)
    return lr, coef, d, gout


def _select(coef, s, compact):
    idx = oracle.dict_select(coef, s)
    return idx, np.take_along_axis(coef, idx.astype(np.int64), 1) if compact else coef


def _check(got, want, mags, c, k, dtype, pixels):
    chain = 2 * (k * k + c + 16) + 16
    gc, gd, gg = (None if x is None else host(x).astype(np.float64) for x in got)
    if gc is not None:
        bound = chain * U32 * mags[0]
        if dtype == "f16":
            bound = bound + (np.abs(want[0]) + bound) * U16 + 2.0 ** -25
        assert np.isfinite(gc).all() and np.all(np.abs(gc - want[0]) <= bound + 1e-30), np.max(np.abs(gc - want[0]) / (bound + 1e-30))
    sums = chain + 160 + pixels / 128 / 16           # (fewer blocks than 16 would only be used for fewer tiles)
    for g, w, m in ((gd, want[1], mags[1]), (gg, want[2], mags[2])):
        if g is not None:
            assert np.isfinite(g).all() and np.all(np.abs(g - w) <= sums * U32 * m + 1e-30), np.max(np.abs(g - w) / (sums * U32 * m + 1e-30))
            assert np.linalg.norm(g - w) <= 2e-6 * np.linalg.norm(m) + 1e-30        # a random sign per rounding: far inside


DENSE = [
    # n, c, h, w, r, D, k, dtype
    (1, 3, 64, 64, 2, 72, 5, "f32"), (1, 3, 64, 64, 2, 72, 5, "f16"),
    (2, 3, 33, 50, 4, 72, 5, "f16"), (1, 3, 20, 67, 3, 72, 5, "f16"), (1, 3, 30, 35, 4, 72, 5, "f16"), (1, 3, 30, 34, 4, 72, 5, "f16"),
    (1, 1, 40, 24, 2, 16, 3, "f16"), (1, 3, 24, 40, 2, 32, 7, "f16"), (1, 3, 24, 40, 2, 32, 7, "f32"),
    (1, 3, 12, 40, 4, 128, 5, "f16"), (1, 3, 10, 24, 2, 256, 3, "f16"), (1, 3, 10, 24, 2, 256, 3, "f32"), (1, 2, 10, 24, 2, 129, 7, "f16"),
    (1, 5, 9, 16, 2, 7, 9, "f32"), (1, 5, 9, 16, 2, 7, 9, "f16"), (1, 4, 9, 16, 2, 256, 9, "f32"), (1, 9, 8, 8, 1, 12, 5, "f16"),
    (1, 3, 7, 5, 3, 3, 1, "f32"), (1, 3, 8, 8, 1, 3, 1, "f16"), (1, 3, 1, 1, 2, 72, 5, "f16"), (1, 1, 1, 1, 1, 1, 3, "f32"), (1, 1, 1, 1, 8, 1, 5, "f16"),
    (1, 3, 3, 100, 4, 72, 5, "f16"), (1, 1, 300, 1, 8, 24, 5, "f16"), (3, 2, 17, 32, 1, 20, 7, "f16"), (1, 4, 16, 16, 2, 40, 7, "f16"),
    (5, 3, 16, 16, 8, 9, 5, "f16"), (2, 3, 65, 64, 2, 8, 3, "f16"), (1, 3, 130, 40, 2, 65, 5, "f16"), (1, 3, 40, 130, 4, 96, 7, "f16"),
]


@pytest.mark.parametrize("bilinear", [False, True])
@pytest.mark.parametrize("n,c,h,w,r,D,k,dt", DENSE)
def test_dense(n, c, h, w, r, D, k, dt, bilinear):
    lr, coef, d, g = _inputs(n, c, h, w, r, D, k, dt)
    want, mags = train_ref.grads(lr, coef, None, None, d, g, r, k, "dense", bilinear=bilinear)
    got = sr.sr_dict_regress_dense_grad(to(lr), to(coef), to(d), to(g), r, k, sr.SR_UPSAMPLE_BILINEAR if bilinear else 0)
    _check((*got, None), want, mags, c, k, dt, n * h * w * r * r)
    assert sr.sr_device_status() == 0


SELECTED = [
    # n, c, h, w, r, D, k, s, dtype
    (1, 3, 33, 52, 4, 72, 5, 8, "f16"), (1, 3, 33, 51, 4, 72, 5, 8, "f16"), (2, 3, 21, 31, 3, 32, 7, 4, "f16"), (2, 1, 24, 32, 2, 100, 3, 16, "f16"),
    (1, 3, 20, 24, 2, 72, 5, 8, "f32"), (1, 3, 20, 24, 2, 72, 5, 72, "f16"), (1, 3, 20, 24, 2, 72, 5, 1, "f16"), (1, 5, 9, 16, 2, 12, 9, 5, "f16"),
    (1, 3, 8, 16, 4, 256, 5, 20, "f16"), (1, 3, 8, 16, 4, 200, 5, 130, "f16"), (1, 3, 7, 5, 3, 3, 1, 2, "f32"), (1, 3, 1, 1, 1, 4, 3, 4, "f16"), (1, 2, 16, 16, 8, 130, 7, 33, "f16"),
]


@pytest.mark.parametrize("mode", ["listed", "compact", "global", "global compact"])
@pytest.mark.parametrize("n,c,h,w,r,D,k,s,dt", SELECTED)
def test_selected(n, c, h, w, r, D, k, s, dt, mode):
    lr, coef, d, g = _inputs(n, c, h, w, r, D, k, dt, seed=3)
    compact, gamma, flags = mode.endswith("compact"), None, 0
    if mode.startswith("global"):
        idx = np.sort(np.random.default_rng(s).permutation(D)[:s]).astype(np.uint8)
        gamma, flags = signed_gamma(s), sr.SR_IDX_GLOBAL
        coef = np.ascontiguousarray(coef[:, idx.astype(int)]) if compact else coef
    else:
        idx, coef = _select(coef, s, compact)
    flags |= sr.SR_COEF_COMPACT if compact else 0
    want, mags = train_ref.grads(lr, coef, idx, gamma, d, g, r, k, mode.split()[0], compact=compact)
    got = sr.sr_dict_regress_selected_grad(to(lr), to(coef), to(idx), to(gamma), to(d), to(g), r, k, s, flags)
    _check(got, want, mags, c, k, dt, n * h * w * r * r)
    if not compact:          # atoms that are not listed: zeros, not small numbers
        assert np.all(host(got[0])[want[0] == 0.0] == 0.0)
    assert sr.sr_device_status() == 0


@pytest.mark.parametrize("k", [3, 5, 7])
@pytest.mark.parametrize("n,h,w", [(1, 1, 8), (1, 2, 8), (2, 3, 16), (1, 1, 136), (3, 5, 136), (1, 17, 120)])
def test_lists_on_frames_with_fewer_rows_than_a_tile(n, h, w, k):
    lr, coef, d, g = _inputs(n, 3, h, w, 1, 9, k, "f16", seed=h + w)
    idx, coef = _select(coef, 2, False)
    want, mags = train_ref.grads(lr, coef, idx, None, d, g, 1, k, "listed")
    for kw in ({}, {"want_dict": False}, {"want_coef": False}):
        got = sr.sr_dict_regress_selected_grad(to(lr), to(coef), to(idx), None, to(d), to(g), 1, k, 2, **kw)
        have = [i for i in (0, 1) if got[i] is not None]
        full = sr.sr_dict_regress_selected_grad(to(lr), to(coef), to(idx), None, to(d), to(g), 1, k, 2)
        _check([got[i] if i in have else full[i] for i in (0, 1)] + [None], want, mags, 3, k, "f16", n * h * w)
    assert sr.sr_device_status() == 0


def test_subset_without_reweights_in_any_order_and_with_an_atom_twice():
    lr, coef, d, g = _inputs(1, 3, 16, 24, 2, 24, 5, "f16", seed=4)
    for idx, gamma in (([9, 3, 17], None), ([5, 2, 5, 11], [0.5, 1.5, -2.0, 1.0]), ([7], [0.0])):
        idx, gamma = np.array(idx, np.uint8), None if gamma is None else np.array(gamma, np.float32)
        want, mags = train_ref.grads(lr, coef, idx, gamma, d, g, 2, 5, "global")
        got = sr.sr_dict_regress_selected_grad(to(lr), to(coef), to(idx), to(gamma), to(d), to(g), 2, 5, len(idx), sr.SR_IDX_GLOBAL)
        assert (got[2] is None) == (gamma is None)
        _check(got, want, mags, 3, 5, "f16", 16 * 24 * 4)


@pytest.mark.parametrize("dt", ["f16", "f32"])
def test_against_differences_of_the_forward_pass(dt):
    """L(coef, dict) = sum(grad_out * out) is linear in each argument: its difference along a direction is the gradient's inner product
    with the direction, up to rounding, at any step size."""
    n, c, h, w, r, D, k, s = 1, 3, 14, 20, 3, 24, 5, 5
    lr, coef, d, g = _inputs(n, c, h, w, r, D, k, dt, seed=6)
    rng = np.random.default_rng(8)
    coef2 = (coef.astype(np.float64) + rng.normal(0, 0.1, coef.shape)).astype(coef.dtype)
    d2 = (d + rng.normal(0, 0.1, d.shape)).astype(np.float32)
    idx = oracle.dict_select(coef, s)
    sub, gam, gam2 = np.array([1, 4, 6, 13, 20], np.uint8), signed_gamma(5), signed_gamma(5, seed=10)
    L = lambda out: float((out * g.astype(np.float64)).sum())  # noqa: E731
    dense = lambda cf, di: L(oracle.dict_regress_dense(lr, cf, di, r, k))  # noqa: E731
    listed = lambda cf, di: L(oracle.dict_regress_selected(lr, cf, idx, None, di, r, k, s))  # noqa: E731
    subset = lambda cf, di, ga=gam: L(oracle.dict_regress_selected(lr, cf, sub, ga, di, r, k, s, flags=oracle.IDX_GLOBAL))  # noqa: E731
    args = to(lr), to(coef)
    for f, got in ((dense, sr.sr_dict_regress_dense_grad(*args, to(d), to(g), r, k)),
                   (listed, sr.sr_dict_regress_selected_grad(*args, to(idx), None, to(d), to(g), r, k, s)),
                   (subset, sr.sr_dict_regress_selected_grad(*args, to(sub), to(gam), to(d), to(g), r, k, s, sr.SR_IDX_GLOBAL))):
        gc, gd = host(got[0]).astype(np.float64), host(got[1]).astype(np.float64)
        dc, dd = coef2.astype(np.float64) - coef, d2.astype(np.float64) - d
        eps = U16 if dt == "f16" else 64 * U32
        assert abs((gc * dc).sum() - (f(coef2, d) - f(coef, d))) <= eps * np.abs(gc * dc).sum() + 2.0 ** -25 * np.abs(dc).sum()
        assert abs((gd * dd).sum() - (f(coef, d2) - f(coef, d))) <= 1e-5 * np.abs(gd * dd).sum()
    dg = gam2.astype(np.float64) - gam
    assert abs((host(got[2]) * dg).sum() - (subset(coef, d, gam2) - subset(coef, d))) <= 1e-5 * np.abs(host(got[2]) * dg).sum()


@pytest.mark.parametrize("w", [32, 31])
def test_parts_buffers_and_repetition(w):
    lr, coef, d, g = (to(a) for a in _inputs(1, 3, 30, w, 4, 72, 5, "f16", seed=2))
    both = sr.sr_dict_regress_dense_grad(lr, coef, d, g, 4, 5)
    gc, none = sr.sr_dict_regress_dense_grad(lr, coef, d, g, 4, 5, want_dict=False)
    assert none is None and torch.equal(gc, both[0])
    none, gd = sr.sr_dict_regress_dense_grad(lr, coef, d, g, 4, 5, want_coef=False)
    assert none is None and torch.equal(gd, both[1])
    # the caller's buffers, full of NaN before, and a scratch of the size asked for
    from paper_2303_08999_b200 import api
    import ctypes
    need = sr.load_library().sr_dict_regress_grad_scratch_bytes(ctypes.byref(api.sr_dims(1, 3, 30, w, 4, 5, 72)))
    bufs = [torch.full_like(x, float("nan")) for x in both] + [torch.full((need,), 255, dtype=torch.uint8, device="cuda")]
    again = sr.sr_dict_regress_dense_grad(lr, coef, d, g, 4, 5, grad_coef=bufs[0], grad_dict=bufs[1], scratch=bufs[2])
    assert again[0] is bufs[0] and torch.equal(bufs[0], both[0]) and torch.equal(bufs[1], both[1])
    with pytest.raises(sr.SrError):
        sr.sr_dict_regress_dense_grad(lr, coef, d, g, 4, 5, scratch=bufs[2][:need - 16])
    with pytest.raises(ValueError):
        sr.sr_dict_regress_selected_grad(lr, coef, None, None, d, g, 4, 5, 8)
    with pytest.raises(ValueError):
        sr.sr_dict_regress_dense_grad(lr, coef, d, g[:, :2].contiguous(), 4, 5)


@pytest.mark.parametrize("shift", [1, 4, 8])
def test_tensors_at_odd_addresses_and_neighbours_untouched(shift):
    """Slices of larger buffers: 2- and 8-byte aligned coefficients (the general path) and 16-byte aligned ones; what lies around the
    outputs stays."""
    lr, coef, d, g = _inputs(1, 3, 20, 32, 4, 40, 5, "f16", seed=5)
    want, mags = train_ref.grads(lr, coef, None, None, d, g, 4, 5, "dense")

    def inside(a, fill):
        buf = torch.full((a.size + 64,), fill, dtype=torch.from_numpy(a[:0]).dtype, device="cuda")
        view = buf[shift: shift + a.size].view(a.shape)
        return buf, view
    cbuf, cview = inside(coef, float("nan"))
    cview.copy_(to(coef))
    gbuf, gview = inside(coef, 7.0)
    got = sr.sr_dict_regress_dense_grad(to(lr), cview, to(d), to(g), 4, 5, grad_coef=gview)
    _check((*got, None), want, mags, 3, 5, "f16", 80 * 128)
    assert bool((gbuf[:shift] == 7).all()) and bool((gbuf[shift + coef.size:] == 7).all())


def test_dictionaries_and_gradients_far_from_one():
    """Nothing on the way may leave the range of binary16: tiny and huge gradients, atoms and images, and atoms of very different size."""
    for g_scale, d_scale, u_scale in ((1e-12, 1.0, 1.0), (1e8, 1e-6, 1.0), (1e-3, 1e5, 1e-4), (1.0, 1.0, 255.0), (1e-20, 1e10, 1e6), (1e20, 1e-12, 1e-6)):
        lr, coef, d, g = _inputs(1, 3, 24, 32, 2, 40, 5, "f32", seed=7)
        d = d * np.float32(d_scale)
        d[::3] *= np.float32(1e-3)
        lr, g = lr * np.float32(u_scale), g * np.float32(g_scale)
        for dt in (np.float32, np.float16):
            cf = coef.astype(dt)
            want, mags = train_ref.grads(lr, cf, None, None, d, g, 2, 5, "dense")
            got = sr.sr_dict_regress_dense_grad(to(lr), to(cf), to(d), to(g), 2, 5)
            top = 65504.0 if dt == np.float16 else 3e38
            inside = np.abs(want[0]) * 1.01 < top                     # (a gradient beyond binary16 is Inf: the caller's loss scale)
            gc = np.where(inside, host(got[0]).astype(np.float64), want[0])
            _check((torch.from_numpy(gc), got[1], None), want, mags, 3, 5, "f16" if dt == np.float16 else "f32", 48 * 64)
    # (zeros everywhere)
    z = sr.sr_dict_regress_dense_grad(to(lr), to(cf), to(d), torch.zeros_like(to(g)), 2, 5)
    assert not z[0].any() and not z[1].any()


@pytest.mark.parametrize("dt,w", [("f16", 32), ("f16", 31), ("f32", 32)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_values_that_are_not_finite_stay_with_their_pixels_and_atoms(dt, w, bad):
    r, k = 4, 5
    lr, coef, d, g = _inputs(1, 3, 20, w, r, 24, k, dt, seed=9)
    clean = [host(x) for x in sr.sr_dict_regress_dense_grad(to(lr), to(coef), to(d), to(g), r, k)]
    # a pixel's incoming gradient
    g2 = g.copy()
    g2[0, 1, 37, 50] = bad
    gc, gd = (host(x) for x in sr.sr_dict_regress_dense_grad(to(lr), to(coef), to(d), to(g2), r, k))
    hit = np.zeros(gc.shape[2:], bool)
    hit[37, 50] = True
    assert not np.isfinite(gc[0, :, hit]).any() and not np.isfinite(gd).any()
    same = gc[0][:, ~hit].astype(np.float64) - clean[0][0][:, ~hit]
    assert np.abs(same).max() <= 1e-3 * np.abs(clean[0]).max()         # (their rounding may move with the tile's scale, nothing else)
    # one coefficient: its atom's row alone
    c2 = coef.copy()
    c2[0, 5, 30, 31] = bad
    gc, gd = (host(x) for x in sr.sr_dict_regress_dense_grad(to(lr), to(c2), to(d), to(g), r, k))
    assert np.array_equal(gc, clean[0]) and not np.isfinite(gd[5]).any()
    others = np.arange(24) != 5
    assert np.array_equal(gd[others], clean[1][others])
    # under a list that leaves it out it does not count at all
    idx = np.broadcast_to(np.array([1, 2, 9], np.uint8).reshape(1, 3, 1, 1), (1, 3) + coef.shape[2:]).copy()
    a = sr.sr_dict_regress_selected_grad(to(lr), to(coef), to(idx), None, to(d), to(g), r, k, 3)
    b = sr.sr_dict_regress_selected_grad(to(lr), to(c2), to(idx), None, to(d), to(g), r, k, 3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # an LR pixel reaches the HR pixels whose patches read it
    l2 = lr.copy()
    l2[0, 0, 10, 12] = bad
    gc, _ = (host(x) for x in sr.sr_dict_regress_dense_grad(to(l2), to(coef), to(d), to(g), r, k))
    far = np.ones(gc.shape[2:], bool)
    far[10 * r - 3 * r - 2: 10 * r + 4 * r + 2, 12 * r - 3 * r - 2: 12 * r + 4 * r + 2] = False
    assert np.isfinite(gc[0][:, far]).all() and not np.isfinite(gc[0][:, 10 * r, 12 * r]).any()
    assert np.abs(gc[0][:, far].astype(np.float64) - clean[0][0][:, far]).max() <= 1e-3 * np.abs(clean[0]).max()


def test_index_beyond_the_dictionary_is_held_to_the_last_atom():
    lr, coef, d, g = _inputs(1, 3, 16, 16, 2, 20, 5, "f16", seed=11)
    idx = oracle.dict_select(coef[:, :19], 3)
    idx[0, 0] = 200
    held = np.minimum(idx, 19)
    args = (to(lr), to(coef)), (None, to(d), to(g), 2, 5, 3)
    a = sr.sr_dict_regress_selected_grad(*args[0], to(idx), *args[1])
    b = sr.sr_dict_regress_selected_grad(*args[0], to(held), *args[1])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("mode", ["dense", "listed", "global"])
def test_streams_and_graph_replay(mode):
    data = [_inputs(1, 3, 32, 48, 4, 72, 5, "f16", seed=20 + i) for i in range(3)]
    d, idx = to(data[0][2]), None
    if mode == "listed":
        idx = [to(_select(x[1], 8, False)[0]) for x in data]
    if mode == "global":
        idx = [torch.arange(0, 72, 9, dtype=torch.uint8, device="cuda")] * 3
    gamma = torch.linspace(0.5, 1.5, 8, device="cuda") if mode == "global" else None

    def call(lr, coef, g, ix):
        if mode == "dense":
            return sr.sr_dict_regress_dense_grad(lr, coef, d, g, 4, 5)
        return sr.sr_dict_regress_selected_grad(lr, coef, ix, gamma, d, g, 4, 5, 8, sr.SR_IDX_GLOBAL if mode == "global" else 0)
    ins = [(to(x[0]), to(x[1]), to(x[3]), None if idx is None else idx[i].clone()) for i, x in enumerate(data)]
    want = [[None if t is None else t.clone() for t in call(*a)] for a in ins]
    static = [None if t is None else t.clone() for t in ins[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = call(*ins[1])
    side.synchronize()
    assert all(a is None or torch.equal(a, b) for a, b in zip(on_side, want[1]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call(*static)
    for i in (2, 1):
        for t, a in zip(static, ins[i]):
            if t is not None:
                t.copy_(a)
        graph.replay()
        torch.cuda.synchronize()
        assert all(a is None or torch.equal(a, b) for a, b in zip(outs, want[i]))
    assert sr.sr_device_status() == 0


@pytest.mark.parametrize("w", [632, 636, 634, 633])          # TMA, copies of 8 and 4 bytes, single elements
@pytest.mark.parametrize("k,D,c", [(3, 16, 3), (5, 72, 3), (7, 40, 1), (5, 128, 4), (7, 128, 3), (5, 200, 3)])
@pytest.mark.parametrize("mode", ["dense", "listed", "compact", "global", "global compact"])
def test_frames_of_many_tiles_a_block(w, k, D, c, mode):
    """Every ring of the pipelines wraps many times: 1.2 million pixels, every element of both gradients against fp64 on the device."""
    n, h, s, compact = 3, 640, 6, mode.endswith("compact")
    gen = torch.Generator(device="cuda").manual_seed(D + k + w)
    lr = torch.rand((n, c, h, w), device="cuda", generator=gen)
    coef = torch.empty((n, D, h, w), device="cuda", dtype=torch.float16).normal_(1 / D, 0.05, generator=gen)
    g = torch.empty((n, c, h, w), device="cuda").normal_(0, 0.05, generator=gen)
    d = torch.empty((D, k * k), device="cuda").normal_(0, 0.2, generator=gen)
    idx = gamma = None
    flags = sr.SR_COEF_COMPACT if compact else 0
    if mode in ("listed", "compact"):
        idx = sr.sr_dict_select(coef, s)
        coef = torch.gather(coef, 1, idx.long()).contiguous() if compact else coef
    elif mode != "dense":
        idx = torch.randperm(D, device="cuda", generator=gen)[:s].to(torch.uint8)
        gamma = torch.empty(s, device="cuda").uniform_(0.5, 1.5, generator=gen)
        coef, flags = coef[:, idx.long()].contiguous() if compact else coef, flags | sr.SR_IDX_GLOBAL
    if mode == "dense":
        gc, gd = sr.sr_dict_regress_dense_grad(lr, coef, d, g, 1, k)
        again = sr.sr_dict_regress_dense_grad(lr, coef, d, g, 1, k)
        alone = (sr.sr_dict_regress_dense_grad(lr, coef, d, g, 1, k, want_dict=False)[0], sr.sr_dict_regress_dense_grad(lr, coef, d, g, 1, k, want_coef=False)[1])
    else:
        call = lambda **kw: sr.sr_dict_regress_selected_grad(lr, coef, idx, gamma, d, g, 1, k, s, flags, **kw)  # noqa: E731
        gc, gd, gg = call()
        again, alone = call(), (call(want_dict=False)[0], call(want_coef=False)[1])
    assert sr.sr_device_status() == 0
    assert torch.equal(gc, again[0]) and torch.equal(gd, again[1])                   # the same bits on every run
    p, atoms = (k - 1) // 2, d.double()
    if gamma is not None:
        atoms = d[idx.long()].double() * gamma.double().view(-1, 1)
    A, worst, magnitude = torch.zeros_like(atoms), [0.0, 0.0], 0.0
    for f in range(n):                                                               # scale 1: the image itself
        pad = torch.nn.functional.pad(lr[f:f + 1].double(), (p, p, p, p), mode="replicate")[0]
        G = torch.stack([(pad[:, a:a + h, b:b + w] * g[f].double()).sum(0) for a in range(k) for b in range(k)], -1)
        full = torch.einsum("hwj,lj->lhw", G, atoms)
        bound = torch.einsum("hwj,lj->lhw", G.abs(), atoms.abs())
        weights = coef[f].double()
        if mode == "listed":
            keep = torch.zeros_like(weights).scatter_(0, idx[f].long(), 1.0)
            full, weights = full * keep, weights * keep
        elif mode == "compact":
            weights = torch.zeros((D, h, w), dtype=torch.float64, device="cuda").scatter_(0, idx[f].long(), weights)
            full, bound = torch.gather(full, 0, idx[f].long()), torch.gather(bound, 0, idx[f].long())
        elif mode == "global":
            at = idx.long()
            weights = weights[at]
            spread = torch.zeros((D, h, w), dtype=torch.float64, device="cuda")
            full, bound = spread.index_copy(0, at, full), spread.index_copy(0, at, bound)
        for i, got in enumerate((gc, alone[0])):                                     # |.| of the terms bounds every rounding (see the top of this file)
            worst[i] = max(worst[i], float(((got[f].double() - full).abs() / (full.abs() * U16 + (2 * (k * k + c + 16) + 16) * 2 * U32 * bound + 2.0 ** -25)).max()))
        A += torch.einsum("lhw,hwj->lj", weights, G)
        magnitude = magnitude + torch.einsum("lhw,hwj->lj", weights.abs(), G.abs())
    assert worst[0] <= 1.0 and worst[1] <= 1.0, worst
    want = A
    if gamma is not None:
        want = torch.zeros((D, k * k), dtype=torch.float64, device="cuda").index_copy(0, idx.long(), A * gamma.double().view(-1, 1))
        assert float((gg.double() - (d[idx.long()].double() * A).sum(1)).norm()) <= 2e-6 * float((d[idx.long()].double().abs() * magnitude).sum(1).norm())
    for got in (gd, alone[1]):
        assert float((got.double() - want).norm()) <= 2e-6 * float(magnitude.norm())


@pytest.mark.parametrize("k,D,s", [(3, 72, 8), (5, 72, 8), (5, 72, 21), (5, 128, 8), (5, 17, 3), (7, 72, 8), (7, 32, 16)])
def test_lists_masked_in_place_and_lists_gathered_are_the_same(k, D, s):
    """Lists on four bytes and lists on an odd address take different ways through the kernel. Full frames, every gradient alone and both,
    lists with atoms twice and indices behind the last atom."""
    n, c, h, w, r = 1, 3, 270, 482, 4
    gen = torch.Generator(device="cuda").manual_seed(100 * k + D + s)
    lr = torch.rand((n, c, h, w), device="cuda", generator=gen)
    coef = torch.empty((n, D, h * r, w * r), device="cuda", dtype=torch.float16).normal_(1 / D, 0.05, generator=gen)
    g = torch.empty((n, c, h * r, w * r), device="cuda").normal_(0, 0.05, generator=gen)
    d = torch.empty((D, k * k), device="cuda").normal_(0, 0.2, generator=gen)
    idx = torch.randint(0, D + 4, (n, s, h * r, w * r), device="cuda", dtype=torch.uint8, generator=gen)
    odd = torch.empty(idx.numel() + 1, device="cuda", dtype=torch.uint8)[1:].view(idx.shape)
    odd.copy_(idx)
    call = lambda i, **kw: sr.sr_dict_regress_selected_grad(lr, coef, i, None, d, g, r, k, s, **kw)[:2]  # noqa: E731
    gc, gd = call(odd)
    for _ in range(3):
        for got, want in zip(call(idx) + call(idx, want_dict=False)[:1] + call(idx, want_coef=False)[1:], (gc, gd, gc, gd)):
            assert torch.equal(got, want) if got.dim() == 4 else float((got - want).norm()) <= 2e-6 * float(want.norm())
    assert sr.sr_device_status() == 0
    listed = torch.zeros((D, h * r, w * r), device="cuda", dtype=torch.bool).scatter_(0, idx[0].long().clamp_(max=D - 1), True)
    assert bool((gc[0][~listed] == 0).all()) and bool((gc[0][listed] != 0).float().mean() > 0.99)


@pytest.mark.parametrize("case", ["dense", "listed", "more atoms", "odd width"])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_clean(case):
    """One product's completion is never announced (the hook of the forward calls): the block gives up, nothing hangs, the status says so."""
    D, w = (160, 64) if case == "more atoms" else (40, 33 if case == "odd width" else 64)
    lr, coef, d, g = (to(a) for a in _inputs(1, 3, 24, w, 1 if case == "odd width" else 2, D, 5, "f16", seed=13))
    r = 1 if case == "odd width" else 2
    idx = sr.sr_dict_select(coef, 4) if case == "listed" else None

    def call():
        if idx is not None:
            return sr.sr_dict_regress_selected_grad(lr, coef, idx, None, d, g, r, 5, 4)[:2]
        return sr.sr_dict_regress_dense_grad(lr, coef, d, g, r, 5)
    before = [t.clone() for t in call()]
    assert sr.sr_device_status() == 0
    old = sr.sr_set_wait_limit(2_000_000)
    try:
        sr.sr_test_lose_arrival(1)
        call()
        assert sr.sr_device_status() == 6 and sr.sr_device_status() == 0             # SR_ERR_TIMEOUT, once
    finally:
        sr.sr_test_lose_arrival(0)
        sr.sr_set_wait_limit(old)
    assert all(torch.equal(a, b) for a, b in zip(call(), before)) and sr.sr_device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "f16"])
@pytest.mark.parametrize("D,k", [(72, 5), (24, 9)])
def test_a_call_that_reads_what_the_call_before_it_writes(dt, D, k):
    """The dictionary's gradient alone, for coefficients that the call before on the stream is still writing (another call's grad_coef)."""
    lr, coef, d, g = (to(a) for a in _inputs(2, 3, 90, 120, 4, D, k, dt, seed=17))
    made, first = torch.empty_like(coef), None
    for wait in (True, False, False, False):
        made.zero_()
        torch.cuda.synchronize()
        sr.sr_dict_regress_dense_grad(lr, coef, d, g, 4, k, grad_coef=made, want_dict=False)
        if wait:
            torch.cuda.synchronize()
        gd = sr.sr_dict_regress_dense_grad(lr, made, d, g, 4, k, want_coef=False)[1]
        first = gd.clone() if first is None else first
        assert torch.equal(gd, first)


def test_two_calls_at_once_with_a_scratch_each():
    data = [tuple(to(a) for a in _inputs(2, 3, 60, 80, 4, 72, 5, "f16", seed=40 + i)) for i in range(2)]
    want = [[t.clone() for t in sr.sr_dict_regress_dense_grad(*x, 4, 5)] for x in data]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (st, x) in enumerate(zip(streams, data)):
            with torch.cuda.stream(st):
                got[i].append(sr.sr_dict_regress_dense_grad(*x, 4, 5))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in (0, 1) for run in got[i] for a, b in zip(run, want[i]))
    assert sr.sr_device_status() == 0


def test_full_size_frames_on_sampled_pixels_and_every_atom():
    """The headline frame and a batch whose element offsets pass 2^31: grad_coef at pixels on both sides of the tiles' seams, all of
    grad_dict, against fp64 on the device."""
    for n, h, w, r, D in ((1, 270, 480, 4, 72), (4, 1080, 1920, 2, 72)):
        c, k, H, W = 3, 5, h * r, w * r
        gen = torch.Generator(device="cuda").manual_seed(5)
        lr = torch.rand((n, c, h, w), device="cuda", generator=gen)
        coef = torch.empty((n, D, H, W), device="cuda", dtype=torch.float16).normal_(1 / D, 0.05, generator=gen)
        g = torch.empty((n, c, H, W), device="cuda").normal_(0, 0.05, generator=gen)
        d = to(signed_asymmetric_dictionary(sr_inputs.make_dictionary(D, k)))
        gc, gd = sr.sr_dict_regress_dense_grad(lr, coef, d, g, r, k)
        want_d, worst = torch.zeros((D, k * k), device="cuda", dtype=torch.float64), 0.0
        for f in range(n):
            u = sr.sr_bicubic_upsample(lr[f:f + 1].contiguous(), r).double()         # parity of its own within 2e-6
            pad = torch.nn.functional.pad(u, (2, 2, 2, 2), mode="replicate")[0]
            G = torch.stack([(pad[:, a:a + H, b:b + W] * g[f].double()).sum(0) for a in range(k) for b in range(k)], -1)
            for rows in torch.arange(H, device="cuda").split(240):
                want_d += torch.einsum("lhw,hwj->lj", coef[f][:, rows].double(), G[rows])
            ys = torch.tensor([0, 1, 7, 8, 15, 16, 17, 31, 32, H // 2, H - 17, H - 2, H - 1], device="cuda")
            xs = torch.tensor([0, 1, 63, 64, 127, 128, 129, 255, 256, W // 2, W - 129, W - 2, W - 1], device="cuda")
            want_c = torch.einsum("hwj,lj->lhw", G[ys][:, xs], d.double())
            worst = max(worst, float(((gc[f][:, ys][:, :, xs].double() - want_c).abs() / (want_c.abs() * U16 * 1.01 + 2e-6)).max()))
        assert worst <= 1.0 and bool(torch.isfinite(gc).all())
        assert float((gd.double() - want_d).norm() / want_d.norm()) <= 5e-6
        del lr, coef, g, gc
