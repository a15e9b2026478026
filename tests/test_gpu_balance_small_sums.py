"""The balance loss's gradient where a pixel's coefficients are very small but their sum is a normal number: the gradient is weight / sum
times something of the size of the slopes, finite although weight / sum alone may not be.

Bounds as in test_gpu_balance: the sum of D magnitudes, its reciprocal, the mean slope and the product are a chain of at most D + 8 fp32
roundings on each side of the difference slope - mean. A product of a slope (times the weight) with a magnitude is rounded to a multiple
of 2^-149 where it is subnormal: D of these, half a step each, against a sum of at least 2^-126.
"""
import numpy as np
import pytest

import oracle
import paper_2303_08999_b200 as sr
import train_ref
from gpu_util import host
from train_ref import U32, to

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W", [24, 23])
@pytest.mark.parametrize("size,weight", [(1e-3, 1.0), (1e-3, -65536.0 * 480), (1e-20, 4.8), (1e-20, 65536.0 * 480), (1e-30, 1.0), (1e-30, -65536.0 * 480),
                                         (1e-34, 1.0), (1e-34, 480.0), (1e-34, 65536.0), (1e-36, 1.0), (1e-36, 4.8), (1e-36, -480.0), (2e-38, 1.0), (2e-38, 48.0)])
def test_sums_near_the_smallest_normal_number(size, weight, W):
    rng = np.random.default_rng(3)
    D = 24
    coef = (rng.uniform(0.1, 1.0, (1, D, 20, W)) * rng.choice([-1, 1], (1, D, 20, W)) * size / D).astype(np.float32)
    coef[:, :3] *= 3
    idx = oracle.dict_select(coef, 4)
    _, _, _, slope, gradient, total, p = train_ref.balance(coef, idx, None, False)
    got = sr.sr_select_balance(to(coef), to(idx))
    assert np.all(np.abs(host(got[3]) - slope) <= 2 * U32 * slope)
    want = gradient(weight)
    grad = host(sr.sr_select_balance_grad(to(coef), got[3], None, weight)).astype(np.float64)
    a = slope[:, :, None, None]
    mag = abs(weight) * (a + (a * p).sum(1, keepdims=True)) / total
    # subnormal products: D roundings of 2^-150 in the sum, divided by the sum for the mean and again for the gradient
    bound = (2 * D + 24) * U32 * mag + D * 2.0 ** -150 / total ** 2
    inside = mag < 3e38                                              # (fp32 holds no larger terms)
    assert inside.mean() > 0.9
    bound = np.where(total < np.finfo(np.float32).tiny, 0.0, bound)
    assert np.isfinite(grad[inside]).all() and np.all(np.abs(grad - want)[inside] <= bound[inside])
    start = rng.normal(0, 1, coef.shape).astype(np.float32) * np.float32(np.abs(want[inside]).max())
    added = host(sr.sr_select_balance_grad(to(coef), got[3], None, weight, flags=sr.SR_GRAD_ADD, grad_coef=to(start.copy()))).astype(np.float64)
    want = want + start
    inside &= np.abs(want) < 3e38
    bound = bound + 2 * U32 * np.abs(want)
    assert np.all(np.abs(added - want)[inside] <= bound[inside])


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("dt,W", [("f32", 24), ("f16", 24), ("f32", 23), ("f16", 23)])
def test_a_weight_that_is_not_finite_stays_with_the_pixels_that_count(dt, W, bad):
    """An overflowed loss scale: pixels that do not count (masked, or with a sum of zero) are zero, or keep their bits, all the same."""
    rng = np.random.default_rng(5)
    coef = rng.uniform(0.1, 1.0, (2, 24, 20, W)).astype(np.float16 if dt == "f16" else np.float32)
    coef[1, :, 3, 2:9] = 0
    mask = np.ones((2, 20, W), np.uint8)
    mask[0, 5:, 7:] = 0
    mask[1, :, ::3] = 0
    idx = oracle.dict_select(coef, 4)
    slope = sr.sr_select_balance(to(coef), to(idx), to(mask))[3]
    off = np.broadcast_to(((mask == 0) | (np.abs(coef).sum(1) == 0))[:, None], coef.shape)
    loss_grad = to(np.array([bad], np.float32))
    start = rng.normal(0, 1, coef.shape).astype(coef.dtype)
    for kw in ({"weight": 2.0, "grad_loss": loss_grad}, {"weight": float(bad)}):
        grad = host(sr.sr_select_balance_grad(to(coef), slope, to(mask), **kw))
        assert not np.any(grad[off]) and not np.isfinite(grad[~off]).any()
        grad = host(sr.sr_select_balance_grad(to(coef), slope, to(mask), flags=sr.SR_GRAD_ADD, grad_coef=to(start.copy()), **kw))
        assert np.array_equal(grad[off], start[off]) and not np.isfinite(grad[~off]).any()
