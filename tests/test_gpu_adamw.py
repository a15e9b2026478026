"""The AdamW step over many tensors against fp64, for every parameter, gradient and state type, with odd sizes and addresses, empty
tensors, more tensors than one launch takes, a step count and a rate on the device, and a step that is skipped.

Bounds (32 bits): m, v are two products and a sum, three half-steps each of their terms' magnitudes; the parameter's update is
lr m / (sqrt(v) c + eps) with at most 12 roundings, and p's own two. 8 bits: a stored value is its fp32 value rounded to e4m3
(half a step, 2^-4 relative, or half of the smallest step 2^-10 of the scale), the scale the block's largest magnitude / 448.
"""
import math

import pytest
import torch

import paper_2303_08999_b200 as sr
import train_ref
from train_ref import U16, U32

pytestmark = pytest.mark.gpu

HALF_STEP = {torch.float32: 0.0, torch.float16: U16, torch.bfloat16: 2.0 ** -8}
OPTS = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
SIZES = [1, 2, 7, 8, 9, 255, 256, 257, 0, 1800, 2048, 2049, 4095, 20001]


def _tensors(sizes, ptype, gtype, seed=1, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def one(n, dtype, std, positive=False):
        buf = torch.zeros(n + 32, dtype=dtype, device="cuda")
        x = torch.empty(n, device="cuda").normal_(0, std, generator=gen)
        view = buf[shift: shift + n]
        view.copy_(x * x if positive else x)
        return view
    return ([one(n, ptype, 0.5) for n in sizes], [one(n, gtype, 1.0) for n in sizes], [one(n, torch.float32, 0.1) for n in sizes],
            [one(n, torch.float32, 0.7, True) for n in sizes])


def _check32(before, after, t, opts, grad_scale=1.0):
    for (p, g, m, v), (p2, m2, v2) in zip(before, after):
        wp, wm, wv = train_ref.adamw(p, g, m, v, t, grad_scale=grad_scale, **opts)
        gs = g.double().abs() * abs(grad_scale)
        assert bool(((m2.double() - wm).abs() <= 4 * U32 * (m.double().abs() + gs) + 1e-38).all())
        assert bool(((v2.double() - wv).abs() <= 6 * U32 * (v.double() + gs * gs) + 1e-38).all())
        den = (wv / (1 - opts["beta2"] ** t)).sqrt() + opts["eps"]
        step = opts["lr"] / (1 - opts["beta1"] ** t) * (m.double().abs() + gs) / den
        bound = 16 * U32 * step + 3 * U32 * p.double().abs()
        bound = bound + HALF_STEP[p.dtype] * (wp.abs() + bound) + (2.0 ** -25 if p.dtype == torch.float16 else 0.0)
        assert bool(((p2.double() - wp).abs() <= bound + 1e-38).all())


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("gtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("ptype", [torch.float32, torch.float16, torch.bfloat16])
def test_states_in_32_bits(ptype, gtype, shift):
    p, g, m, v = _tensors(SIZES, ptype, gtype, shift=shift)
    plan = sr.sr_adamw_plan(p, m, v)
    for t in (1, 2, 1000):
        before = [[x.clone() for x in row] for row in zip(p, g, m, v)]
        sr.sr_adamw_step(plan, g, t, grad_scale=0.25, **OPTS)
        _check32(before, list(zip(p, m, v)), t, OPTS, 0.25)


def _decode(code, scale, n):
    return code.float().double() * scale.double().repeat_interleave(sr.ADAMW_BLOCK)[:n]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("ptype,gtype", [(torch.float32, torch.float32), (torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)])
def test_states_in_8_bits(ptype, gtype, shift):
    sizes = SIZES
    p, g, _, _ = _tensors(sizes, ptype, gtype, seed=2, shift=shift)
    for x in g:                                               # gradients of very different size within a block
        x.mul_(torch.logspace(-4, 1, max(1, x.numel()), device="cuda")[: x.numel()].to(x.dtype))
    g[3].zero_()
    f8 = torch.float8_e4m3fn
    state = [[torch.zeros(n + 32, dtype=f8, device="cuda")[shift: shift + n] for n in sizes] for _ in range(2)]
    scale = [[torch.zeros((n + 255) // 256, device="cuda") for n in sizes] for _ in range(2)]
    plan = sr.sr_adamw_plan(p, *state, *scale)
    for t in (1, 2, 3):
        before = [x.clone() for x in p]
        old = [[_decode(c, s, c.numel()) for c, s in zip(state[i], scale[i])] for i in (0, 1)]
        sr.sr_adamw_step(plan, g, t, **OPTS)
        for i, n in enumerate(sizes):
            if n == 0:
                continue
            wp, wm, wv = train_ref.adamw(before[i], g[i], old[0][i], old[1][i] ** 2, t, **OPTS)
            root, blocks = wv.sqrt(), (n + 255) // 256
            pad = lambda x: torch.nn.functional.pad(x, (0, blocks * 256 - n)).view(blocks, 256)  # noqa: E731
            for code, sc, want in ((state[0][i], scale[0][i], wm), (state[1][i], scale[1][i], root)):
                top = pad(want.abs()).amax(1)
                assert bool(((sc.double() * 448 - top).abs() <= 8 * U32 * top + 1e-38).all())
                held = _decode(code, sc, n)
                grid = sc.double().repeat_interleave(256)[:n]
                # half a step of e4m3 (and the value's own rounding before it); the smallest root is held up instead of rounded down
                bound = want.abs() * (2.0 ** -4 + 1e-5) + grid * 2.0 ** -10 * 1.0001
                small = (want > 0) & (want < grid * 2.0 ** -10)
                if code is state[1][i]:
                    bound = torch.where(small, grid * 2.0 ** -9, bound)
                    assert bool((held[(want > 0) & (grid > 0)] > 0).all())
                assert bool(((held - want).abs() <= bound + 1e-38).all())
            den = (wv / (1 - OPTS["beta2"] ** t)).sqrt() + OPTS["eps"]
            step = OPTS["lr"] / (1 - OPTS["beta1"] ** t) * (old[0][i].abs() + g[i].double().abs()) / den
            bound = 24 * U32 * step + 3 * U32 * before[i].double().abs()
            bound = bound + HALF_STEP[ptype] * (wp.abs() + bound) + (2.0 ** -25 if ptype == torch.float16 else 0.0)
            assert bool(((p[i].double() - wp).abs() <= bound + 1e-38).all())
    assert not scale[0][3].any() and not state[0][3].float().any()              # nothing moved: still the fresh state


def test_8_bit_blocks_of_tiny_values():
    """Scales among the subnormals, where dividing by 448 loses bits: codes stay in range, nothing turns into NaN."""
    for size in (1e-36, 1e-38, 1e-41, 1e-44):
        n = 300
        p, g = [torch.zeros(n, device="cuda")], [torch.full((n,), size, device="cuda")]
        state = [torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
        scale = [torch.zeros(2, device="cuda") for _ in range(2)]
        plan = sr.sr_adamw_plan(p, [state[0]], [state[1]], [scale[0]], [scale[1]])
        for t in (1, 2):
            sr.sr_adamw_step(plan, g, t, 1e-3)
        assert bool(torch.isfinite(p[0]).all()) and all(bool(torch.isfinite(s.float()).all()) for s in state)


def test_more_tensors_than_one_launch_takes():
    sizes = [1 + (i * 37) % 700 for i in range(1000)]
    p, g, m, v = _tensors(sizes, torch.float32, torch.float32, seed=3)
    before = [[x.clone() for x in row] for row in zip(p, g, m, v)]
    launches = sr.sr_launch_count()
    sr.sr_adamw_step(sr.sr_adamw_plan(p, m, v), g, 5, **OPTS)
    assert 2 <= sr.sr_launch_count() - launches <= 4
    _check32(before, list(zip(p, m, v)), 5, OPTS)


def test_what_lies_between_the_tensors_stays():
    buf = [torch.full((1000,), 5.0, device="cuda") for _ in range(4)]
    views = [[b[17:300], b[301:307], b[600:999]] for b in buf]
    sr.sr_adamw_step(sr.sr_adamw_plan(views[0], views[2], views[3]), views[1], 1, 1e-2)
    hit = torch.zeros(1000, dtype=torch.bool, device="cuda")
    hit[17:300], hit[301:307], hit[600:999] = True, True, True
    for b in (buf[0], buf[2], buf[3]):
        assert bool((b[~hit] == 5).all())
    assert bool((buf[0][hit] != 5).all()) and bool((buf[3][hit] != 5).all())      # (m: 0.9 * 5 + 0.1 * 5 is 5)
    assert bool((buf[1] == 5).all())


def test_rate_step_and_skip_on_the_device_in_a_replayed_graph():
    p, g, m, v = _tensors([1800, 333], torch.float32, torch.float32, seed=4)
    q, _, qm, qv = ([x.clone() for x in row] for row in (p, g, m, v))
    plan, host_plan = sr.sr_adamw_plan(p, m, v), sr.sr_adamw_plan(q, qm, qv)
    lr, step, skip = torch.tensor([1e-3], device="cuda"), torch.tensor([1], device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    opts = {k: OPTS[k] for k in ("beta1", "beta2", "eps", "weight_decay")}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_adamw_step(plan, g, step, lr, skip=skip, **opts)
    for t, rate in ((1, 1e-3), (2, 5e-3), (3, 1e-2), (10000, 1e-3), (10001, 1e-4)):
        step.fill_(t)
        lr.fill_(rate)
        for x in g:
            x.mul_(1.5).add_(0.1)
        graph.replay()
        sr.sr_adamw_step(host_plan, g, t, rate, **opts)
        for a, b in zip(p, q):                                # the two forms differ in how the corrections are rounded
            assert torch.allclose(a, b, rtol=1e-6, atol=8 * U32 * rate * 10)
        assert all(torch.equal(a, b) for a, b in zip(m + v, qm + qv))
    skip.fill_(1)
    old = [x.clone() for x in p + m + v]
    for x in g:
        x.fill_(math.nan)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(old, p + m + v))


def test_plan_follows_replaced_storage_and_refuses_other_tensors():
    p, g, m, v = _tensors([100, 50], torch.float32, torch.float32, seed=5)
    plan = sr.sr_adamw_plan(p, m, v)
    sr.sr_adamw_step(plan, g, 1, 1e-3)
    fresh = torch.zeros(100, device="cuda")
    old = p[0].clone()
    kept = p[0].data
    p[0].data = fresh
    sr.sr_adamw_step(plan, g, 2, 1e-3)
    assert bool(fresh.any()) and torch.equal(kept, old)
    p[0].data = torch.zeros(101, device="cuda")
    with pytest.raises(ValueError):
        sr.sr_adamw_step(plan, g, 3, 1e-3)
    p[0].data = fresh
    with pytest.raises(ValueError):
        sr.sr_adamw_step(plan, g[:1], 3, 1e-3)
    with pytest.raises(TypeError):
        sr.sr_adamw_step(plan, [g[0], g[1].half()], 3, 1e-3)
    with pytest.raises(TypeError):
        sr.sr_adamw_step(plan, [g[0], g[1].cpu()], 3, 1e-3)
    with pytest.raises(TypeError):
        sr.sr_adamw_step(plan, [g[0], torch.zeros(100, device="cuda")[::2]], 3, 1e-3)
    with pytest.raises(sr.SrError):
        sr.sr_adamw_step(plan, g, 0, 1e-3)
    with pytest.raises(ValueError):
        sr.sr_adamw_plan(p, [m[1], m[0]], v)
    with pytest.raises(TypeError):
        sr.sr_adamw_plan(p, [x.half() for x in m], v)
