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
