"""What a plan of the AdamW step follows and what it refuses when its parameters are given other data."""
import pytest
import torch

import paper_2303_08999_b200 as sr

pytestmark = pytest.mark.gpu


def _plan(p):
    return sr.sr_adamw_plan([p], [torch.zeros(p.numel(), device="cuda")], [torch.zeros(p.numel(), device="cuda")])


@pytest.mark.parametrize("view,error", [(lambda x: x[:50], ValueError), (lambda x: x.view(torch.float16)[:100], TypeError), (lambda x: x.view(4, 25).t(), TypeError),
                                        (lambda x: x.view(10, 10).t(), TypeError), (lambda x: x.view(torch.int32), TypeError)])
def test_another_view_of_the_same_memory_is_refused(view, error):
    """It starts at the parameter's address, so the address alone does not tell (all of it lies in the parameter's own memory)."""
    memory = torch.arange(100, dtype=torch.float32, device="cuda")
    p = memory.view(100)
    plan = _plan(p)
    g = torch.ones(100, device="cuda")
    sr.sr_adamw_step(plan, [g], 1, 1e-3)
    before = memory.clone()
    p.data = view(memory)
    assert p.data_ptr() == memory.data_ptr()
    with pytest.raises(error):
        sr.sr_adamw_step(plan, [g], 2, 1e-3)
    assert torch.equal(memory, before)
    p.data = memory.view(4, 25)                          # another shape is the same elements in the same order
    sr.sr_adamw_step(plan, [g], 2, 1e-3)
    assert bool((memory != before).all())


def test_new_memory_at_the_old_address_is_checked():
    """A freed address is what the allocator gives next: a parameter of half the bytes would be written past its end."""
    p = torch.zeros(1 << 20, device="cuda")
    plan = _plan(p)
    p.data = torch.zeros(1, device="cuda")
    p.data = torch.zeros(1 << 20, dtype=torch.float16, device="cuda")
    with pytest.raises(TypeError):
        sr.sr_adamw_step(plan, [torch.ones(1 << 20, device="cuda")], 1, 1e-3)
    p.data = torch.zeros(1 << 19, device="cuda")
    with pytest.raises(ValueError):
        sr.sr_adamw_step(plan, [torch.ones(1 << 20, device="cuda")], 1, 1e-3)


def test_a_plan_refuses_any_one_tensor_that_does_not_fit():
    """A list is checked as a whole: whichever place the wrong tensor is at, and whichever list, it is found."""
    def lists(bits):
        n = [300] * 5
        state = (lambda: [torch.zeros(x, device="cuda") for x in n]) if bits == 32 else (lambda: [torch.zeros(x, dtype=torch.float8_e4m3fn, device="cuda") for x in n])
        out = [[torch.zeros(x, device="cuda") for x in n], state(), state()]
        return out if bits == 32 else out + [[torch.zeros(2, device="cuda") for _ in n] for _ in range(2)]
    for bits in (32, 8):
        sr.sr_adamw_plan(*lists(bits))
        for which in range(3 if bits == 32 else 5):
            for place in (0, 2, 4):
                for change, error in ((lambda t: t.cpu(), TypeError), (lambda t: t.to(torch.float64), TypeError), (lambda t: torch.cat([t, t])[::2], TypeError),
                                      (lambda t: torch.cat([t, t]), ValueError), (lambda t: t[:-1], ValueError)):
                    given = lists(bits)
                    given[which][place] = change(given[which][place].float()).to(given[which][place].dtype) if error is ValueError else change(given[which][place])
                    with pytest.raises(error):
                        sr.sr_adamw_plan(*given)


def test_a_plan_keeps_the_memory_of_its_states():
    p, m, v = torch.zeros(1 << 18, device="cuda"), torch.zeros(1 << 18, device="cuda"), torch.zeros(1 << 18, device="cuda")
    plan = sr.sr_adamw_plan([p], [m], [v])
    addresses = {m.data_ptr(), v.data_ptr()}
    m.data, v.data = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    del m, v
    others = [torch.full((1 << 18,), 7.0, device="cuda") for _ in range(8)]            # what the allocator would put there
    assert not addresses & {t.data_ptr() for t in others}
    sr.sr_adamw_step(plan, [torch.ones_like(p)], 1, 1e-3)
    assert all(bool((t == 7).all()) for t in others) and bool((p < 0).all())


@pytest.mark.parametrize("place", [0, 1])
def test_a_parameter_without_a_gradient_is_refused_by_name(place):
    p = [torch.zeros(10, device="cuda"), torch.zeros(20, device="cuda")]
    plan = sr.sr_adamw_plan(p, [torch.zeros_like(x) for x in p], [torch.zeros_like(x) for x in p])
    g = [torch.ones_like(x) for x in p]
    g[place] = None
    with pytest.raises(TypeError, match="needs a gradient"):
        sr.sr_adamw_step(plan, g, 1, 1e-3)
    assert not p[0].any() and not p[1].any()
