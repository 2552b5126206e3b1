"""AdamW where sqrt(v) is of the order of a small eps, down to v that is subnormal."""

import numpy as np
import pytest

import adamw_ref as R
from test_gpu_adamw import host

pytestmark = pytest.mark.gpu

SHAPES = [(64, 512), (9, 257), (1000,)]
B1, B2, EPS = 0.9, 0.999, 1e-30


def cases(shape):
    """Gradients whose squares times 1 - b2 go from fp32's smallest numbers to well above its subnormals."""
    k = int(np.prod(shape))
    # 2^-73 squared times 2^-10 is 2^-156, nothing in fp32; 2^-45 squared 2^-100
    return np.ldexp(1.0 + np.arange(k) % 7 / 8, -73 + np.arange(k) % 29).astype(np.float32) * np.where(np.arange(k) % 2, 1, -1)


@pytest.mark.parametrize("rank", [0, 4])
@pytest.mark.parametrize("bits", [32, 8])
def test_small_values(bits, rank):
    import torch
    from paper_2306_08881_amd.adamw import AdamW
    gs = []
    for s in SHAPES:
        g = cases(s).astype(np.float32)
        n, m = R.matrix(s)
        if rank:  # a row's gradients are multiples of the first row's: a product without rounding
            a, b = np.zeros((n, rank), np.float32), np.zeros((m, rank), np.float32)
            a[:, 1] = np.ldexp(1.0, np.arange(n) % 3)
            b[:, 1] = g[:m]
            gs.append((a, b))
        else:
            gs.append(g)
    p = [torch.zeros(s, device="cuda") for s in SHAPES]
    opt = AdamW(SHAPES, p, bits=bits, seed=1)
    opt.set_grads([tuple(torch.from_numpy(x).cuda() for x in g) if rank else torch.from_numpy(g).cuda() for g in gs])
    opt.step(1, lr=1.0, betas=(B1, B2), eps=EPS, weight_decay=0.0)
    b1, c1, b2, c2 = (np.float32(x) for x in (B1, 1 - B1, B2, 1 - B2))
    for x, g in zip(p, gs):
        g = (g[0][:, 1:2] * g[1][:, 1]).reshape(-1) if rank else g
        # the moments as fp32 has them, operation by operation, subnormal numbers included
        m, v = g * c1, (g * g) * c2
        assert (v == 0).any() and ((v > 0) & (v < 2.0 ** -126)).any() and (v > 2.0 ** -110).any()
        den = np.sqrt(v.astype(np.float64)) / np.sqrt(1 - B2) + EPS
        want = -m.astype(np.float64) / (1 - B1) / den
        # the root 2 ulp; rs, the denominator's sum, the reciprocal (1 ulp), the quotient, the factor and the
        # last sum: 10 half units and some
        got = host(x).reshape(-1)
        assert (np.abs(got - want) <= 14 * R.U * np.abs(want)).all(), np.max(np.abs(got / want - 1))


def test_small_state_of_8_bits():
    """Steps on an 8-bit state whose v is subnormal: the update stays of the order of one."""
    import torch
    from paper_2306_08881_amd.adamw import AdamW
    p = torch.zeros(4, 600, device="cuda")
    opt = AdamW([(4, 600)], [p], bits=8, seed=2)
    g = torch.full((4, 600), 1e-18, device="cuda")
    opt.set_grads([g])
    for t in range(1, 6):
        before = p.clone()
        opt.step(t, lr=1.0, betas=(B1, B2), eps=EPS, weight_decay=0.0)
        # equal values take the top code of their block, exactly; constant gradients make steps of -1: m and
        # sqrt(v) are right to within the moments' roundings (v near 1e-39 has units of 2^-149, 1.4e-6 of it)
        assert bool(((p - before) + 1).abs().max() < 1e-4), t
