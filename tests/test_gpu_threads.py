"""Calls of several host threads at once, on a stream each: calls of different sizes share kernels, and none may disturb what another
one has set for its launch. The threads call the C entry points themselves, so that the interpreter holds them up as little as possible."""
import ctypes
import threading

import pytest
import torch

import paper_2303_08999_b200 as sr
from gpu_util import on_kernel
from paper_2303_08999_b200 import api

pytestmark = pytest.mark.gpu


def _at_once(jobs, calls):
    """Every job (a function of a stream's handle that makes one call and returns its status) `calls` times, a thread each."""
    failed, start = [], threading.Barrier(len(jobs))

    def work(job, stream):
        start.wait()
        for _ in range(calls):
            status = job(stream.cuda_stream)
            if status:
                failed.append(status)
    threads = [threading.Thread(target=work, args=(job, torch.cuda.Stream())) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return failed


def _problem(D, k, dtype=torch.float32, hw=8):
    gen = torch.Generator(device="cuda").manual_seed(D)
    one = lambda *shape: torch.rand(shape, device="cuda", generator=gen)  # noqa: E731
    return one(1, 3, hw, hw), one(1, D, hw, hw).to(dtype), one(D, k * k), one(1, 3, hw, hw), api.sr_dims(1, 3, hw, hw, 1, k, D)


@pytest.mark.parametrize("k,sizes", [(5, (72, 128, 72, 128)), (9, (48, 72, 256, 24)), (3, (80, 256, 100, 256))])
def test_fp32_gradients_of_different_sizes(k, sizes):
    lib, jobs, outs = sr.load_library(), [], []
    for D in sizes:
        lr, coef, d, g, dims = _problem(D, k)
        want = sr.sr_dict_regress_dense_grad(lr, coef, d, g, 1, k)
        gc, gd = torch.empty_like(coef), torch.empty_like(d)
        scratch = torch.empty(lib.sr_dict_regress_grad_scratch_bytes(ctypes.byref(dims)), dtype=torch.uint8, device="cuda")
        outs.append((want, (gc, gd)))
        jobs.append(lambda st, a=(lr, coef, d, g, gc, gd, scratch), dims=dims: lib.sr_dict_regress_dense_grad(
            a[0].data_ptr(), a[1].data_ptr(), api.SR_F32, a[2].data_ptr(), a[3].data_ptr(), a[4].data_ptr(), a[5].data_ptr(), ctypes.byref(dims), 0,
            a[6].data_ptr(), a[6].numel(), st))
    torch.cuda.synchronize()
    assert _at_once(jobs, 4000) == []
    assert all(torch.equal(x, y) for want, got in outs for x, y in zip(want, got))


def test_general_regressions_of_different_sizes():
    """9 x 9 atoms, whose dictionary is the largest that the general kernel holds: 160 to 256 atoms, a size of shared memory each."""
    lib, jobs, outs = sr.load_library(), [], []
    with on_kernel(0):
        for D in (160, 200, 240, 256):
            lr, coef, d, _, dims = _problem(D, 9)
            want = sr.sr_dict_regress_dense(lr, coef, d, 1, 9)
            out = torch.empty_like(want)
            outs.append((want, out))
            jobs.append(lambda st, a=(lr, coef, d, out), dims=dims: lib.sr_dict_regress_dense(
                a[0].data_ptr(), a[1].data_ptr(), api.SR_F32, a[2].data_ptr(), a[3].data_ptr(), ctypes.byref(dims), 0, st))
        torch.cuda.synchronize()
        assert _at_once(jobs, 4000) == []
    assert all(torch.equal(want, got) for want, got in outs)
