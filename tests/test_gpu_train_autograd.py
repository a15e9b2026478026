"""Tensors that the training-side calls change in place count as changed: a backward pass that saved one of them refuses, as it does after
PyTorch's own changes in place, instead of using what stands there now."""
import pytest
import torch

import paper_2303_08999_b200 as sr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_between_forward_and_backward(bits):
    w, b = torch.full((300,), 2.0, device="cuda", requires_grad=True), torch.zeros(5, device="cuda", requires_grad=True)
    state = [[torch.zeros(t.numel(), dtype=torch.float32 if bits == 32 else torch.float8_e4m3fn, device="cuda") for t in (w, b)] for _ in range(2)]
    scales = [] if bits == 32 else [[torch.zeros((t.numel() + 255) // 256, device="cuda") for t in (w, b)] for _ in range(2)]
    plan = sr.sr_adamw_plan([w, b], *state, *scales)
    loss = (w * w).sum() + b.sum()
    sr.sr_adamw_step(plan, [torch.ones_like(w), torch.ones_like(b)], 1, 1e-2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    assert w.grad is None
    grads = torch.autograd.grad((w * w).sum() + b.sum(), [w, b])             # a forward pass after the step is an ordinary one
    assert torch.equal(grads[0], 2 * w.detach()) and bool((grads[1] == 1).all())
    with torch.no_grad():
        before = w._version
        sr.sr_adamw_step(plan, [x.contiguous() for x in grads], 2, 1e-2)
    assert w._version > before


def test_gradients_written_or_added_to_a_tensor():
    D, k = 8, 3
    lr, coef, d, g = torch.rand(1, 1, 8, 8, device="cuda"), torch.rand(1, D, 8, 8, device="cuda"), torch.rand(D, k * k, device="cuda"), torch.rand(1, 1, 8, 8, device="cuda")
    idx = sr.sr_dict_select(coef, 2)
    slope = sr.sr_select_balance(coef, idx)[3]
    sub, gamma = torch.tensor([1, 4], dtype=torch.uint8, device="cuda"), torch.ones(2, device="cuda")
    gc, gd, gg = torch.zeros_like(coef), torch.zeros_like(d), torch.zeros(2, device="cuda")
    for call, written in ((lambda: sr.sr_dict_regress_dense_grad(lr, coef, d, g, 1, k, grad_coef=gc, grad_dict=gd), (gc, gd)),
                          (lambda: sr.sr_dict_regress_selected_grad(lr, coef, idx, None, d, g, 1, k, 2, grad_coef=gc, grad_dict=gd), (gc, gd)),
                          (lambda: sr.sr_dict_regress_selected_grad(lr, coef, sub, gamma, d, g, 1, k, 2, sr.SR_IDX_GLOBAL, grad_coef=gc, grad_dict=gd, grad_gamma=gg), (gc, gd, gg)),
                          (lambda: sr.sr_select_balance_grad(coef, slope, grad_coef=gc), (gc,)),
                          (lambda: sr.sr_select_balance_grad(coef, slope, flags=sr.SR_GRAD_ADD, grad_coef=gc), (gc,))):
        before = [t._version for t in written]
        read = [t._version for t in (lr, coef, d, g, idx, slope)]
        call()
        assert all(t._version > v for t, v in zip(written, before))
        assert [t._version for t in (lr, coef, d, g, idx, slope)] == read
    x = torch.ones_like(gc, requires_grad=True)
    loss = (x * gc).sum()                                    # saves gc
    sr.sr_select_balance_grad(coef, slope, flags=sr.SR_GRAD_ADD, grad_coef=gc)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():                             # such tensors have no versions
        sr.sr_select_balance_grad(coef, slope, grad_coef=torch.zeros_like(coef))
