"""Balance loss of a selection and its gradient against the fp64 definition, with masks that leave nothing, pixels whose coefficients
are zero, values that are not finite in masked places, odd sizes and addresses, and differences of the loss.

Bounds: a pixel's sum of D magnitudes, its reciprocal and a share are a chain of at most D + 4 fp32 operations, all of one sign, so
shares are right to (D + 4) half-steps; a block's sum of shares adds its pixels per lane (at most all pixels of a small frame / 32) and 5
more. The gradient takes the difference slope - mean, each off by (D + 8) half-steps of its own size.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2303_08999_b200 as sr
import train_ref
from gpu_util import host
from train_ref import U16, U32, to

pytestmark = pytest.mark.gpu


def _inputs(n, D, H, W, s, dt, masked, seed=1):
    rng = np.random.default_rng(seed)
    coef = rng.normal(1.0 / D, 0.05, (n, D, H, W)).astype(np.float16 if dt == "f16" else np.float32)
    coef[:, : max(1, D // 8)] *= 3
    mask = None
    if masked:
        mask = np.zeros((n, H, W), np.uint8)
        for f in range(n):
            mask[f, : rng.integers(1, H + 1), : rng.integers(1, W + 1)] = 1 + f % 255
    return coef, oracle.dict_select(coef, s), mask


def _check(coef, idx, mask, per_frame, weight, dt, grad_loss=None, start=None):
    loss, counts, share, slope, gradient, total, p = train_ref.balance(coef, idx, mask, per_frame)
    n, D, H, W = coef.shape
    got = sr.sr_select_balance(to(coef), to(idx), to(mask), sr.SR_BALANCE_PER_FRAME if per_frame else 0)
    assert np.array_equal(host(got[1]), counts)
    pixels = min(H * W / 32, 256) + 16
    assert np.all(np.abs(host(got[2]) - share) <= (D + 8 + pixels) * U32 * share + 1e-30)
    assert np.all(np.abs(host(got[3]) - slope) <= 2 * U32 * slope)
    assert abs(host(got[0])[0] - loss) <= (D + 8 + pixels) * U32 * loss
    grad = to(start.copy()) if start is not None else None
    grad = sr.sr_select_balance_grad(to(coef), got[3], to(mask), weight, grad_loss, sr.SR_GRAD_ADD if start is not None else 0, grad)
    w = weight * (1.0 if grad_loss is None else float(grad_loss))
    want = gradient(w)
    a = slope[:, :, None, None]
    mag = abs(w) * (a + (a * p).sum(1, keepdims=True)) / total
    on = np.ones((n, 1, H, W), bool) if mask is None else mask[:, None] != 0
    by_definition = ~on | (coef == 0) | (np.abs(np.where(on, coef, 1)).sum(1, keepdims=True, dtype=np.float64) < np.finfo(np.float32).tiny)
    bound = (2 * D + 24) * U32 * np.where(by_definition, 0.0, mag)       # (elsewhere a zero is slope - mean, each with its roundings)
    if start is not None:
        want = want + start.astype(np.float64)
        bound = bound + U32 * np.abs(want)
    if dt == "f16":
        bound = bound + np.abs(want) * U16 * 1.001 + 2.0 ** -25
    assert np.all(np.abs(host(grad).astype(np.float64) - want) <= bound + 1e-38), np.max(np.abs(host(grad) - want) / (bound + 1e-38))
    return got, grad


CASES = [
    # n, D, H, W, s, dtype
    (1, 72, 64, 64, 8, "f16"), (1, 72, 64, 64, 8, "f32"), (2, 72, 37, 53, 8, "f16"), (3, 72, 37, 53, 8, "f32"), (1, 32, 128, 128, 4, "f16"),
    (1, 1, 5, 7, 1, "f16"), (1, 2, 1, 1, 1, "f32"), (4, 16, 9, 16, 16, "f16"), (1, 17, 40, 24, 3, "f16"), (1, 33, 31, 8, 2, "f32"), (1, 48, 16, 16, 5, "f16"),
    (1, 81, 24, 24, 6, "f16"), (1, 128, 20, 24, 16, "f16"), (2, 129, 11, 24, 20, "f32"), (1, 256, 24, 24, 40, "f16"), (1, 256, 23, 23, 256, "f32"),
    (300, 8, 3, 5, 2, "f16"), (1, 72, 1, 3001, 8, "f16"), (1, 72, 700, 600, 8, "f16"),
]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("per_frame", [False, True])
@pytest.mark.parametrize("n,D,H,W,s,dt", CASES)
def test_balance(n, D, H, W, s, dt, per_frame, masked):
    coef, idx, mask = _inputs(n, D, H, W, s, dt, masked)
    start = np.random.default_rng(4).normal(0, 0.5, coef.shape).astype(coef.dtype)
    _check(coef, idx, mask, per_frame, 0.01 * n * H * W, dt)
    _, grad = _check(coef, idx, mask, per_frame, -0.5 * n * H * W, dt, grad_loss=torch.tensor([2.0], device="cuda"), start=start)
    if masked:                    # pixels that do not count keep their bits
        off = np.broadcast_to(mask[:, None] == 0, coef.shape)
        assert np.array_equal(host(grad)[off], start[off])


def test_masks_that_leave_nothing_zero_pixels_and_what_stands_in_masked_places():
    coef, idx, _ = _inputs(3, 24, 20, 24, 4, "f16", False)
    mask = np.zeros((3, 20, 24), np.uint8)
    for per_frame in (False, True):
        got, grad = _check(coef, idx, mask, per_frame, 100.0, "f16")              # nothing at all
        assert float(got[0]) == 0.0 and not got[1].any() and not grad.any()
        mask[1, 3:9, 5:] = 1
        got, grad = _check(coef, idx, mask, per_frame, 100.0, "f16")              # one frame of three
        bad, badidx = coef.copy(), idx.copy()
        off = mask == 0
        bad.transpose(0, 2, 3, 1)[off] = np.array([np.nan, np.inf, -np.inf, 65504] * 6, np.float16)
        badidx.transpose(0, 2, 3, 1)[off] = 255
        again = sr.sr_select_balance(to(bad), to(badidx), to(mask), sr.SR_BALANCE_PER_FRAME if per_frame else 0)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        assert torch.equal(sr.sr_select_balance_grad(to(bad), again[3], to(mask), 100.0), grad)
        mask[1] = 0
    for dt in ("f16", "f32"):
        coef, idx, _ = _inputs(1, 24, 20, 24, 4, dt, False)
        coef[0, :, 4:9, 3:11] = 0                                                 # sums of zero share equally and have no gradient
        coef[0, 5] = 0
        _check(coef, idx, None, False, 500.0, dt)
    tiny = np.full((1, 8, 4, 8), 1e-42, np.float32)                               # a sum below the smallest normal number
    _check(tiny, oracle.dict_select(tiny, 2), None, False, 1.0, "f32")


def test_indices_beyond_the_dictionary_are_not_counted():
    coef, idx, _ = _inputs(1, 20, 16, 16, 4, "f16", False)
    idx[0, 2, 3:7] = 20
    idx[0, 1, 9] = 255
    got, _ = _check(coef, idx, None, False, 10.0, "f16")
    assert int(got[1].sum()) == 16 * 16 * 4 - 4 * 16 - 16


def test_even_use_has_loss_one_and_a_collapsed_selection_costs_more():
    D, s, H, W = 16, 2, 16, 16
    coef = np.ones((1, D, H, W), np.float32)
    idx = (np.arange(H * W * s).reshape(1, s, H, W) % D).astype(np.uint8)
    assert abs(float(sr.sr_select_balance(to(coef), to(idx))[0]) - 1.0) < 1e-6
    coef[:, :2] = 20.0
    few = sr.sr_select_balance(to(coef), to(oracle.dict_select(coef, s)))
    assert float(few[0]) > 5.0
    g = host(sr.sr_select_balance_grad(to(coef), few[3]))
    assert (g[:, :2] > 0).all() and (g[:, 2:] < 0).all()                          # a step against it lowers the two and lifts the rest


def test_against_differences_of_the_loss():
    coef, idx, mask = _inputs(2, 24, 12, 16, 4, "f32", True, seed=8)
    rng = np.random.default_rng(3)
    for per_frame in (False, True):
        _, _, _, slope, _, _, _ = train_ref.balance(coef, idx, mask, per_frame)
        g = host(sr.sr_select_balance_grad(to(coef), to(slope.astype(np.float32)), to(mask))).astype(np.float64)
        step = rng.normal(0, 1e-5, coef.shape) * (np.abs(coef) > 1e-4)            # no coefficient changes its sign
        up, down = ((train_ref.balance(coef + e, idx, mask, per_frame)[0]) for e in (step, -step))
        assert abs((g * step).sum() - (up - down) / 2) <= 1e-4 * np.abs(g * step).sum()


@pytest.mark.parametrize("dt,shift", [("f16", 1), ("f16", 4), ("f16", 8), ("f32", 1), ("f32", 4)])
def test_odd_addresses(dt, shift):
    coef, idx, mask = _inputs(1, 40, 16, 24, 4, dt, True)
    buf = to(np.concatenate([coef.reshape(-1)] * 2))
    out = torch.full_like(buf, 3.0)
    cv, gv = buf[shift: shift + coef.size].view(coef.shape), out[shift: shift + coef.size].view(coef.shape)
    cv.copy_(to(coef))
    want = sr.sr_select_balance(to(coef), to(idx), to(mask))
    got = sr.sr_select_balance(cv, to(idx), to(mask))
    assert torch.equal(got[1], want[1]) and torch.equal(got[3], want[3])
    assert torch.allclose(got[2], want[2], rtol=1e-5, atol=0) and torch.allclose(got[0], want[0], rtol=1e-5, atol=0)
    g = sr.sr_select_balance_grad(cv, got[3], to(mask), 50.0, grad_coef=gv)
    ref = sr.sr_select_balance_grad(to(coef), got[3], to(mask), 50.0)
    assert torch.allclose(g.float(), ref.float(), rtol=2 * U16 if dt == "f16" else 1e-5, atol=1e-6)
    assert bool((out[:shift] == 3).all()) and bool((out[shift + coef.size:] == 3).all())


def test_repetition_streams_and_graph_replay():
    data = [_inputs(2, 72, 40, 64, 8, "f16", True, seed=30 + i) for i in range(3)]
    ins = [tuple(to(a) for a in x) for x in data]

    def call(coef, idx, mask):
        loss, counts, share, slope = sr.sr_select_balance(coef, idx, mask)
        return loss, counts, share, slope, sr.sr_select_balance_grad(coef, slope, mask, 100.0)
    want = [[t.clone() for t in call(*a)] for a in ins]
    assert all(torch.equal(a, b) for a, b in zip(call(*ins[0]), want[0]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(*ins[1])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
    static = [t.clone() for t in ins[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call(*static)
    for i in (2, 1, 2):
        for t, a in zip(static, ins[i]):
            t.copy_(a)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))


def test_more_elements_than_32_bits_count():
    n, D, H, W, s = 4, 72, 2160, 3840, 2
    coef = torch.empty((n, D, H, W), dtype=torch.float16, device="cuda").normal_(1 / D, 0.05)
    idx = torch.randint(0, D, (n, s, H, W), dtype=torch.uint8, device="cuda")
    loss, counts, share, slope = sr.sr_select_balance(coef, idx)
    for f in (0, n - 1):
        assert torch.equal(counts[f].long(), torch.bincount(idx[f].flatten().int(), minlength=D))
        p = sum((coef[f][:, r:r + 270].float().abs() / coef[f][:, r:r + 270].float().abs().sum(0)).double().sum((1, 2)) for r in range(0, H, 270)) / (H * W)
        assert float((share[f] - p).abs().max() / p.max()) <= 1e-5
    grad = sr.sr_select_balance_grad(coef, slope, None, 1e6)
    last = coef[n - 1, :, -1, -64:].float()
    p = last.abs() / last.abs().sum(0)
    a = slope[n - 1].view(D, 1)
    want = 1e6 * last.sign() * (a - (a * p).sum(0)) / last.abs().sum(0)
    assert torch.allclose(grad[n - 1, :, -1, -64:].float(), want, rtol=2e-3, atol=1e-6)
