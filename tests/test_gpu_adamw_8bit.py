"""What the 8-bit optimiser states hold: the codes and scales of the formula in fp32, bit for bit, and blocks with a gradient that is not
finite.

The formula in fp32 is `_step` below: every operation rounded once, in the order in which sr.h writes it, as elementary torch operations
do. The kernel's codes and scales have to be the same bits, so there is no tolerance.
"""
import numpy as np
import pytest
import torch

import paper_2303_08999_b200 as sr

pytestmark = pytest.mark.gpu

BLOCK, F8_MAX = 256, 448.0


def _fresh(sizes):
    state = [[torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for n in sizes] for _ in range(2)]
    scale = [[torch.zeros((n + BLOCK - 1) // BLOCK, device="cuda") for n in sizes] for _ in range(2)]
    return state, scale


def _blocks(x):
    blocks = (x.numel() + BLOCK - 1) // BLOCK
    return torch.nn.functional.pad(x, (0, blocks * BLOCK - x.numel())).view(blocks, BLOCK)


def _codes(x, scale):
    return torch.where(scale > 0, x / scale, 0.0).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn).float()


def _step(g, m, v, m_scale, v_scale, beta1, beta2, grad_scale):
    """The states after a step as (m codes, m scales, root codes, root scales), codes as values."""
    g = _blocks(g.float() * grad_scale)
    m = _blocks(m.float()) * m_scale.view(-1, 1)
    root = _blocks(v.float()) * v_scale.view(-1, 1)
    m = m * beta1 + g * (1 - beta1)
    v = root * root * beta2 + g * g * (1 - beta2)
    root = torch.sqrt(v)
    per = torch.tensor(1.0 / F8_MAX, dtype=torch.float32, device="cuda")
    ms, vs = m.abs().amax(1, keepdim=True) * per, root.amax(1, keepdim=True) * per
    held = _codes(root, vs)
    held = torch.where((root > 0) & (held == 0) & (vs > 0), 2.0 ** -9, held)
    return _codes(m, ms), ms.view(-1), held, vs.view(-1)


def _same(got, want, n):
    code_m, scale_m, code_v, scale_v = got
    for code, value in ((code_m, want[0]), (code_v, want[2])):
        a, b = code.float(), value.flatten()[:n]
        differ = int(((a != b) & ~(a.isnan() & b.isnan())).sum())
        assert differ == 0, (differ, n)
    assert torch.equal(scale_m, want[1]) and torch.equal(scale_v, want[3])


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.9, 0.95), (0.0, 0.0)])
@pytest.mark.parametrize("gtype", [torch.float32, torch.float16, torch.bfloat16])
def test_codes_and_scales_are_the_formulas_in_fp32(gtype, beta1, beta2):
    gen = torch.Generator(device="cuda").manual_seed(6)
    sizes = [1, 255, 256, 257, 4099, 300007]
    p = [torch.zeros(n, device="cuda") for n in sizes]
    state, scale = _fresh(sizes)
    plan = sr.sr_adamw_plan(p, *state, *scale)
    for t in (1, 2, 3, 4):
        g = [(torch.empty(n, device="cuda").normal_(generator=gen) * torch.logspace(-6, 3, n, device="cuda")).to(gtype) for n in sizes]
        old = [[x.clone() for x in row] for row in state + scale]
        sr.sr_adamw_step(plan, g, t, 1e-3, beta1, beta2, grad_scale=0.37)
        for i, n in enumerate(sizes):
            _same((state[0][i], scale[0][i], state[1][i], scale[1][i]), _step(g[i], *(row[i] for row in old), beta1, beta2, 0.37), n)


@pytest.mark.parametrize("unit", [1.0, 1e-3, 3e-20, 1e-28, 1e-33, 1e-36, 3e25, 1e31])
def test_values_half_way_between_two_codes(unit):
    """Quotients next to and at the middle of two codes, over many scales: the quotient is rounded once, then to the even code."""
    blocks = 4096
    steps = np.array([s * 2.0 ** e for e in range(-6, 8) for s in (1.0625, 1.1875, 1.3125, 1.4375, 1.5625, 1.6875, 1.8125, 1.9375)] + [0.0009765625, 0.0029296875, 440.0, 432.0])
    rng = np.random.default_rng(5)
    scale = (rng.uniform(1.0, 2.0, blocks) * unit).astype(np.float32)
    x = np.zeros((blocks, BLOCK), np.float32)
    at = (scale[:, None].astype(np.float64) * steps).astype(np.float32)          # the nearest fp32 numbers to the middles, and those beside
    k = steps.size
    x[:, :k], x[:, k:2 * k] = at, -np.nextafter(at, np.float32(np.inf))
    x[:, 255] = scale * np.float32(F8_MAX)
    g = torch.from_numpy(x.reshape(-1)).cuda()
    state, scales = _fresh([g.numel()])
    sr.sr_adamw_step(sr.sr_adamw_plan([torch.zeros_like(g)], *state, *scales), [g], 1, 1e-3, 0.0, 0.9)
    _same((state[0][0], scales[0][0], state[1][0], scales[1][0]),
          _step(g, *(torch.zeros_like(y[0]) for y in state + scales), 0.0, 0.9, 1.0), g.numel())


@pytest.mark.parametrize("gtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n,at,rest", [(1, [0], 0.0), (256, [17], 0.0), (256, [255], 0.5), (256, range(256), 0.0), (300, [299], 0.25), (300, [3], 0.0), (1000, [256, 511], 1.0)])
def test_a_gradient_that_is_not_finite_marks_its_whole_block(n, at, rest, bad, gtype):
    """None of the block's states is finite after the step or after a clean one; the other blocks are those of a step without it."""
    at = list(at)
    hit = torch.zeros((n + BLOCK - 1) // BLOCK, dtype=torch.bool, device="cuda")
    hit[[i // BLOCK for i in at]] = True
    element = hit.repeat_interleave(BLOCK)[:n]
    runs = []
    for value in (0.125, bad):                           # the same run without and with it
        p = [torch.ones(n, device="cuda")]
        state, scale = _fresh([n])
        plan = sr.sr_adamw_plan(p, *state, *scale)
        sr.sr_adamw_step(plan, [torch.full((n,), 0.5, device="cuda", dtype=gtype)], 1, 1e-3)
        g = torch.full((n,), rest, device="cuda", dtype=gtype)
        g[at] = value
        sr.sr_adamw_step(plan, [g], 2, 1e-3)
        runs.append([p[0].clone(), *(c[0].float() * s[0].repeat_interleave(BLOCK)[:n] for c, s in zip(state, scale))])
        sr.sr_adamw_step(plan, [torch.full((n,), 0.5, device="cuda", dtype=gtype)], 3, 1e-3)
        runs[-1] += [p[0], *(c[0].float() * s[0].repeat_interleave(BLOCK)[:n] for c, s in zip(state, scale))]
    clean, got = runs
    for i in (1, 2, 4, 5):                               # the moments after the step and after the next
        assert not torch.isfinite(got[i][element]).any()
        assert torch.equal(got[i][~element], clean[i][~element])
    assert not torch.isfinite(got[0][at]).any() and not torch.isfinite(got[3][element]).any()
    others = torch.ones(n, dtype=torch.bool, device="cuda")
    others[at] = False
    assert torch.equal(got[0][others], clean[0][others]) and torch.equal(got[3][~element], clean[3][~element])
