"""The training-side calls run together as a fine-tuning step: select, regress, the loss's gradient, the regression's gradient, the
balance loss and its gradient on top, and the optimiser's step on the dictionary, the re-weights and the coefficients (which stand for the
network behind them). Each step's results are those of the same step in fp64 from the same starting point."""
import numpy as np
import pytest
import torch

import oracle
import paper_2303_08999_b200 as sr
import sr_inputs
import train_ref
from gpu_util import host, signed_asymmetric_dictionary
from train_ref import to

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eight", [False, True])
def test_fine_tuning_under_a_per_pixel_selection(eight):
    r, k, s, D = 2, 5, 4, 24
    wl = sr_inputs.Workload("t", 2, 3, 24, 32, r, D=D, k=k, coef_dtype="f32")
    lr, d, coef = sr_inputs.make_inputs(wl, seed=77)
    d = signed_asymmetric_dictionary(d)
    target = np.random.default_rng(1).uniform(0, 1, (2, 3, 48, 64)).astype(np.float32)
    t_lr, t_target = to(lr), to(target)
    params = [to(d), to(coef)]
    if eight:
        new = lambda p: torch.zeros(p.numel(), dtype=torch.float8_e4m3fn, device="cuda")  # noqa: E731
        scales = [[torch.zeros((p.numel() + 255) // 256, device="cuda") for p in params] for _ in range(2)]
        plan = sr.sr_adamw_plan(params, [new(p) for p in params], [new(p) for p in params], *scales)
    else:
        plan = sr.sr_adamw_plan(params, [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params])
    for step in (1, 2, 3):
        dict_, coef_ = params
        d0, c0 = host(dict_).copy(), host(coef_).copy()
        m0, v0 = [x.clone() for x in plan.m], [x.clone() for x in plan.v]
        idx = sr.sr_dict_select(coef_, s)
        out = sr.sr_dict_regress_selected(t_lr, coef_, idx, None, dict_, r, k, s)
        g = (out - t_target) * (2.0 / out.numel())
        gc, gd, _ = sr.sr_dict_regress_selected_grad(t_lr, coef_, idx, None, dict_, g, r, k, s)
        loss, counts, share, slope = sr.sr_select_balance(coef_, idx)
        sr.sr_select_balance_grad(coef_, slope, None, 0.01, flags=sr.SR_GRAD_ADD, grad_coef=gc)
        sr.sr_adamw_step(plan, [gd, gc], step, 1e-3)
        # the same in fp64
        widx = oracle.dict_select(c0, s)
        assert np.array_equal(host(idx), widx)
        wg = (oracle.dict_regress_selected(lr, c0, widx, None, d0, r, k, s) - target) * (2.0 / target.size)
        (wc, wd, _), _ = train_ref.grads(lr, c0, widx, None, d0, wg, r, k, "listed")
        wc = wc + train_ref.balance(c0, widx, None, False)[4](0.01)
        for got, want in ((gc, wc), (gd, wd)):
            assert np.linalg.norm(host(got) - want) <= 1e-5 * np.linalg.norm(want)
        for i, (p0, gw) in enumerate(((d0, gd), (c0, gc))):
            if not eight:
                wp, wm, wv = train_ref.adamw(torch.from_numpy(p0).cuda(), gw, m0[i], v0[i], step, 1e-3, 0.9, 0.999, 1e-8, 0.01)
                assert float((params[i].double() - wp).norm()) <= 1e-6 * float(wp.norm())
                assert float((plan.m[i].double() - wm).norm()) <= 1e-6 * float(wm.norm())
            assert bool(torch.isfinite(params[i]).all()) and not np.array_equal(host(params[i]), p0)
    assert sr.sr_device_status() == 0


def test_fine_tuning_after_a_selection_search():
    """Algorithm 1's result (atoms and re-weights) goes into the subset's gradient and the step moves dictionary and re-weights."""
    r, k, D = 2, 5, 24
    wl = sr_inputs.Workload("t", 1, 3, 24, 32, r, D=D, k=k, coef_dtype="f16")
    lr, d, coef = sr_inputs.make_inputs(wl, seed=78)
    d = signed_asymmetric_dictionary(d)
    target = oracle.dict_regress_dense(lr, coef, d, r, k).astype(np.float32)
    t_lr, t_coef, t_d, t_target = (to(a) for a in (lr, coef, d, target))
    G, b, hh = sr.sr_selection_gram(t_lr, t_coef, t_d, t_target, None, r, k)
    idx, gamma, _ = sr.sr_selection_search(G, b, hh, target.size, 0.5, 0.25, 0.05, 1e-4)
    s = idx.numel()
    assert 1 <= s < D
    gamma = gamma.clone()
    plan = sr.sr_adamw_plan([t_d, gamma], [torch.zeros_like(t_d), torch.zeros_like(gamma)], [torch.zeros_like(t_d), torch.zeros_like(gamma)])
    for step in (1, 2):
        d0, g0 = host(t_d).copy(), host(gamma).copy()
        out = sr.sr_dict_regress_selected(t_lr, t_coef, idx, gamma, t_d, r, k, s, sr.SR_IDX_GLOBAL)
        g = (out - t_target) * 64.0
        gc, gd, gg = sr.sr_dict_regress_selected_grad(t_lr, t_coef, idx, gamma, t_d, g, r, k, s, sr.SR_IDX_GLOBAL)
        (wc, wd, wgg), mags = train_ref.grads(lr, coef, host(idx), g0, d0, host(g), r, k, "global")
        for got, want, mag in ((gc, wc, mags[0]), (gd, wd, mags[1]), (gg, wgg, mags[2])):
            assert np.linalg.norm(host(got).astype(np.float64) - want) <= (1e-3 if got is gc else 2e-6) * np.linalg.norm(mag)
        sr.sr_adamw_step(plan, [gd, gg], step, 1e-3)
        outside = np.setdiff1d(np.arange(D), host(idx))
        assert np.allclose(host(t_d)[outside], d0[outside] * (1 - 1e-5), rtol=1e-6, atol=0)      # no gradient: decay alone
    assert sr.sr_device_status() == 0
