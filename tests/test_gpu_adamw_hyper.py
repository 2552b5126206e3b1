"""Hyperparameters at the ends of what the step takes: as fp32, which the kernels compute in."""

import math

import pytest

import adamw_ref as R
from test_gpu_adamw import host

pytestmark = pytest.mark.gpu


def optimiser():
    import torch
    from paper_2306_08881_amd.adamw import AdamW
    p = torch.linspace(-1, 1, 6 * 8, device="cuda").view(6, 8)
    opt = AdamW([(6, 8)], [p])
    opt.set_grads([torch.linspace(1, 2, 6 * 8, device="cuda").view(6, 8)])
    return opt, p


@pytest.mark.parametrize("bad", [dict(eps=1e39), dict(eps=2.0 ** 126 * 1.01), dict(eps=float("inf")), dict(eps=2.0 ** -126 * 0.99),
                                 dict(lr=1e39), dict(lr=1e308), dict(lr=1e38, betas=(0.99999, 0.9)), dict(lr=1e30, weight_decay=1e30),
                                 dict(lr=1e200, weight_decay=1e200), dict(betas=(1 - 1e-9, 0.9)), dict(betas=(0.9, 1 - 1e-9)),
                                 dict(betas=(0.9, 1 - 2.0 ** -25)), dict(betas=(float("nan"), 0.9)), dict(betas=(0.9, float("nan"))),
                                 dict(betas=(0.9, 2.0)), dict(betas=(-1e-9, 0.9))], ids=str)
def test_refused(bad):
    from paper_2306_08881_amd import _lib as L
    opt, p = optimiser()
    before = p.clone()
    with pytest.raises(L.AcpError, match="ACP_E_INVALID"):
        opt.step(**{**dict(step=1, lr=1e-3), **bad})
    assert bool((p == before).all())
    assert float(opt.moments()["m"].abs().max()) == 0.0 and float(opt.moments()["v"].abs().max()) == 0.0


@pytest.mark.parametrize("good", [dict(eps=2.0 ** -126), dict(eps=2.0 ** 126, lr=2.0 ** 100), dict(lr=0.0), dict(lr=1e30),
                                  dict(betas=(0.0, 0.0)), dict(betas=(1 - 2.0 ** -24, 1 - 2.0 ** -24)),
                                  dict(lr=1e-3, weight_decay=1e30)], ids=str)
def test_accepted(good):
    opt, p = optimiser()
    kw = {**R.HYPER, **good}
    before, g = host(p), host(opt._grads[0][0][0])
    opt.step(1, **kw)
    z = 0.0 * before
    want, m, v = R.step(1, before, z, z, g, **kw)
    bp, bm, bv = R.bounds(1, before, z, z, g, z, **kw)
    # the decay factor is rounded by itself, however large it is
    bp = bp + 4 * R.U * abs(1 - kw["lr"] * kw["weight_decay"]) * abs(before)
    assert (abs(host(p) - want) <= bp).all()
    k = before.size
    for name, x, bound in (("m", m, bm), ("v", v, bv)):
        assert (abs(host(opt.moments()[name][:k]).reshape(before.shape) - x) <= bound).all(), name
    assert math.isfinite(float(p.abs().max()))
