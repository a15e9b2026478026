"""Tensors that the training-side calls write and that share memory with another tensor of the call are refused, before anything is written."""
import pytest
import torch

import paper_2303_08999_b200 as sr

pytestmark = pytest.mark.gpu

D, k, s = 8, 3, 2


def _inputs(dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(1)
    one = lambda *shape: torch.rand(shape, device="cuda", generator=gen)  # noqa: E731
    return one(1, 1, 8, 8), one(1, D, 8, 8).to(dtype), one(D, k * k), one(1, 1, 8, 8)


def _refused(call, *tensors):
    before = [t.clone() for t in tensors]
    with pytest.raises(ValueError, match="shares memory"):
        call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, tensors))


def test_gradients_of_the_regression():
    lr, coef, d, g = _inputs()
    idx, both = sr.sr_dict_select(coef, s), torch.zeros(D * 64 + D * 9, device="cuda")
    dense = lambda **kw: sr.sr_dict_regress_dense_grad(lr, coef, d, g, 1, k, **kw)  # noqa: E731
    listed = lambda **kw: sr.sr_dict_regress_selected_grad(lr, coef, idx, None, d, g, 1, k, s, **kw)  # noqa: E731
    for call in (dense, listed):
        _refused(lambda: call(grad_coef=coef), coef)
        _refused(lambda: call(grad_dict=d), d)
        _refused(lambda: call(grad_coef=both[: D * 64].view(coef.shape), grad_dict=both[D * 64 - 1: D * 73 - 1].view(d.shape)), both)
        want = [t.clone() for t in call()[:2]]
        got = call(grad_coef=both[: D * 64].view(coef.shape), grad_dict=both[D * 64:].view(d.shape))           # side by side is apart
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    scratch = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    _refused(lambda: dense(grad_coef=scratch[: D * 256].view(torch.float32).view(coef.shape), scratch=scratch), scratch)
    sub, gamma = torch.tensor([1, 4], dtype=torch.uint8, device="cuda"), torch.ones(2, device="cuda")
    _refused(lambda: sr.sr_dict_regress_selected_grad(lr, coef, sub, gamma, d, g, 1, k, s, sr.SR_IDX_GLOBAL, grad_gamma=gamma), gamma)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_balance_gradient(dtype):
    _, coef, _, _ = _inputs(dtype)
    slope = sr.sr_select_balance(coef, sr.sr_dict_select(coef, s))[3]
    for flags in (0, sr.SR_GRAD_ADD):
        _refused(lambda: sr.sr_select_balance_grad(coef, slope, flags=flags, grad_coef=coef), coef)
    with pytest.raises(ValueError, match="shares memory"):
        sr.sr_select_balance(coef, sr.sr_dict_select(coef, s), scratch=coef.view(torch.uint8))


def test_adamw():
    z = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    p, buf = z(40), z(100)
    for lists in (([p, p], [z(40), z(40)], [z(40), z(40)]), ([p], [p], [z(40)]), ([p], [buf[:40]], [buf[39:79]]), ([buf[:60], buf[50:90]], [z(60), z(40)], [z(60), z(40)])):
        with pytest.raises(ValueError, match="shares memory"):
            sr.sr_adamw_plan(*lists)
    f8 = lambda n: torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda")  # noqa: E731
    scale = z(2)
    with pytest.raises(ValueError, match="shares memory"):
        sr.sr_adamw_plan([z(300)], [f8(300)], [f8(300)], [scale], [scale])
    sr.sr_adamw_plan([z(300), z(0), z(0)], [f8(300), f8(0), f8(0)], [f8(300), f8(0), f8(0)], [z(2), z(0), z(0)], [z(2), z(0), z(0)])
    plan = sr.sr_adamw_plan([buf[:50], buf[50:]], [z(50), z(50)], [z(50), z(50)])                   # side by side is apart
    sr.sr_adamw_step(plan, [torch.ones(50, device="cuda")] * 2, 1, 1e-3)                            # (gradients are read: they may be one tensor)
    assert bool((buf < 0).all())
    q = z(50)
    plan = sr.sr_adamw_plan([q, p], [z(50), z(40)], [z(50), z(40)])
    q.data = buf[10:60]
    p.data = buf[20:60]
    for _ in range(2):                                                                              # (also when it is called again)
        _refused(lambda: sr.sr_adamw_step(plan, [torch.ones(50, device="cuda"), torch.ones(40, device="cuda")], 1, 1e-3), buf)
    q.data = z(50)
    sr.sr_adamw_step(plan, [torch.ones(50, device="cuda"), torch.ones(40, device="cuda")], 1, 1e-3)
