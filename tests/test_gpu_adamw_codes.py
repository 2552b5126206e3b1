"""8-bit moments code by code: the random rounding replayed from its description, in every kernel that does it."""

import numpy as np
import pytest

import adamw_ref as R
from test_gpu_adamw import SHAPES, Problem, given, host

pytestmark = pytest.mark.gpu


def stored(pr, name, i):
    import torch
    st = pr.opt.moments()
    first, blk, blocks, _, _ = pr.opt.tensor_info(i)
    k = int(np.prod(pr.shapes[i]))
    return (st[name][first:first + k].view(torch.uint8).cpu().numpy(), host(st[name + "_scale"][blk:blk + blocks]))


def check_codes(pr, t, seed, c=1.0, **kw):
    """One step; the codes of every tensor against the replay from the state before."""
    import torch
    n = len(pr.shapes)
    before = [(host(pr.p.views[i]), pr.moment("m", i)[0], pr.moment("v", i)[0] ** 2) for i in range(n)]
    grads = [pr.gradient(i) for i in range(n)]
    pr.opt.step(t, **R.HYPER, **kw)
    torch.cuda.synchronize()
    sure = total = 0
    for i in range(n):
        p, m, v = before[i]
        g, dg = grads[i]
        _, m1, v1 = R.step(t, p, m, v, g, c, pr.decay[i], **R.HYPER)
        _, bm, bv = R.bounds(t, p, m, v, g, dg, c, decay=pr.decay[i], **R.HYPER)
        halves = R.random_halves(seed, t, i, np.arange(g.size))
        r1 = np.sqrt(v1)
        br = 0.5 * bv / np.sqrt(np.maximum(v1, 1e-300)) + R.U * r1
        blk = R.block_of(pr.shapes[i])
        for name, x, bx, half in (("m", m1, bm, halves[0]), ("v", r1, br, halves[1])):
            got, scale = stored(pr, name, i)
            scale = scale[blk]
            live = scale > 0
            y = np.abs(x[live]) / scale[live]
            # the scale and its inverse are within 2 ulp of each other's, the product half of one
            dy = bx[live] / scale[live] + 6 * R.U * y
            want, clear = R.codes(y, dy, half[live], name == "v")
            code = got[live] & 127
            wrong = clear & (code != want)
            assert not wrong.any(), (f"tensor {i} {pr.shapes[i]} step {t} {name}: {wrong.sum()} of {clear.sum()} codes, "
                                     f"first at {np.flatnonzero(wrong)[0]}")
            sign = (got[live] >> 7) == 1
            assert (sign == ((x[live] < 0) & (code > 0)))[clear & (np.abs(x[live]) > bx[live]) & (code > 0)].all()
            sure, total = sure + clear.sum(), total + clear.size
    # the replay says something of most codes: bounds of products grow with the rank, and those of rank 256 leave
    # a few hundredths open
    assert sure > 0.9 * total, (sure, total)


@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
@pytest.mark.parametrize("shift,seed", [(0, 0), (1, 2 ** 40 + 7)])
def test_values(grad, shift, seed):
    """Whole-word and ragged rows (k_adamw, both forms)."""
    pr = Problem(SHAPES, 8, grad, shift, copy=shift == 1, seed=seed)
    for t in (1, 2, 1000):
        pr.draw()
        check_codes(pr, t, seed)


@pytest.mark.parametrize("rank", [1, 3, 4, 8, 16, 17, 32, 64, 100, 128, 256])
def test_factors(rank):
    """Block columns of both forms and narrow tiles."""
    pr = Problem(SHAPES, 8, rank=rank, seed=rank)
    for t in (1, 2):
        pr.draw()
        check_codes(pr, t, rank)


def test_joined():
    """Small dense tensors in the products' launch, and narrow tiles in a launch of their own."""
    import torch
    for wide in (True, False):
        shapes = SHAPES if wide else [s for s in SHAPES if R.matrix(s)[1] < 256]
        pr = Problem(shapes, 8, seed=11)
        grads = []
        for i, s in enumerate(shapes):
            n, m = R.matrix(s)
            if i % 2:
                grads.append((torch.randn(n, 8, device="cuda") * 0.1, torch.randn(m, 8, device="cuda") * 0.1))
            else:
                grads.append(torch.randn(n * m, device="cuda") * 1e-2)
        given(pr, grads)
        for t in (1, 2):
            check_codes(pr, t, 11)


def test_large_blocks_of_one_tensor():
    """Tiles of a tensor's middle and end, with blocks that fill their rows and others."""
    pr = Problem([(700, 1100), (700, 1024), (300000,), (9000, 40)], 8, copy=False, seed=5)
    for t in (1, 2):
        pr.draw()
        check_codes(pr, t, 5)


# ---- factors whose product is exact, against the same gradients as values ------------------------------------


def integers(shape, gen, unit=1.0):
    import torch
    return torch.randint(-2, 3, shape, generator=gen, device="cuda").float() * unit


def same_as_values(shapes, bits, rank, steps=2, copy=True):
    """Sums of at most 256 products of integers up to 2 are exact in any order: the whole state, bit for bit."""
    import torch
    from paper_2306_08881_amd.adamw import AdamW
    gen = torch.Generator(device="cuda").manual_seed(rank)
    mats = [R.matrix(s) for s in shapes]
    start = [torch.randn(s, generator=gen, device="cuda") for s in shapes]
    ps = [[x.clone() for x in start] for _ in range(2)]
    cs = [[torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes] if copy else None for _ in range(2)]
    opts = [AdamW(shapes, p, c, bits=bits, seed=rank) for p, c in zip(ps, cs)]
    factors = [[torch.empty(n, rank, device="cuda"), torch.empty(m, rank, device="cuda")] for n, m in mats]
    values = [torch.empty(n * m, device="cuda") for n, m in mats]
    opts[0].set_grads([tuple(f) for f in factors])
    opts[1].set_grads(values)
    for t in range(1, steps + 1):
        for (a, b), g in zip(factors, values):
            a.copy_(integers(a.shape, gen, 2.0 ** -10))
            b.copy_(integers(b.shape, gen))
            for r0 in range(0, a.shape[0], 65536):
                torch.matmul(a[r0:r0 + 65536], b.t(), out=g.view(-1, b.shape[0])[r0:r0 + 65536])
            # the library's product is exact as well
            k = min(50, a.shape[0])
            assert torch.equal(g.view(a.shape[0], -1)[-k:].double().cpu(), a[-k:].double().cpu() @ b.double().cpu().t())
        for o in opts:
            o.step(t, scale=0.5, **R.HYPER)
        torch.cuda.synchronize()
        for i, s in enumerate(shapes):
            assert torch.equal(ps[0][i].view(torch.int32), ps[1][i].view(torch.int32)), (s, t, "p")
            if copy:
                assert torch.equal(cs[0][i].view(torch.int16), cs[1][i].view(torch.int16)), (s, t, "copy")
        moments = [o.moments() for o in opts]
        for name in moments[0]:
            assert torch.equal(moments[0][name].view(torch.uint8), moments[1][name].view(torch.uint8)), (t, name)
    assert float((ps[0][0] - start[0]).abs().max()) > 1e-4


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rank", [1, 2, 3, 4, 8, 15, 16, 17, 24, 32, 33, 64, 100, 128, 129, 200, 256])
def test_exact_products(bits, rank):
    same_as_values(SHAPES, bits, rank)


@pytest.mark.parametrize("rank", [4, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("columns", [1024, 1021, 300])
@pytest.mark.parametrize("copy", [True, False])
def test_exact_products_of_many_rows(rank, columns, copy):
    """So many rows that a tile takes several groups of them at a stride: every row of every tensor."""
    rows = {1024: 70007, 1021: 70007, 300: 140001}[columns]
    # groups of 16 rows by columns of blocks: four tiles' worth and more, where tiles are split from 4096 on
    assert -(-rows // 16) * -(-columns // 256) >= 4 * 4096
    same_as_values([(rows, columns), (33, 1021), (9, 512), (40, 20), (700,)], 8, rank, copy=copy)


@pytest.mark.parametrize("bits", [32, 8])
def test_factors_past_32_bits(bits):
    """A factored tensor of more than 2^32 elements whose gradient is nothing outside its last row."""
    import torch
    from paper_2306_08881_amd.adamw import AdamW
    n, m, rank = (1 << 20) + 5, 4104, 4
    p = torch.zeros(n, m, device="cuda")
    opt = AdamW([(n, m)], [p], bits=bits)
    a, b = torch.zeros(n, rank, device="cuda"), torch.randn(m, rank, device="cuda")
    a[-1] = torch.randn(rank, device="cuda")
    opt.set_grads([(a, b)])
    opt.step(1, **R.HYPER)
    assert int(torch.count_nonzero(p[:-1])) == 0
    x, y = host(a[-1:]), host(b)
    g, dg = (x @ y.T).reshape(-1), ((rank + 1) * R.U * (np.abs(x) @ np.abs(y).T)).reshape(-1)
    z = np.zeros(m)
    want = R.step(1, z, z, z, g, **R.HYPER)[0]
    assert (np.abs(host(p[-1]) - want) <= R.bounds(1, z, z, z, g, dg, **R.HYPER)[0]).all()
    for x in opt.moments().values():  # nothing but the last row's moments and scales either
        cut = (n - 1) * m if x.numel() >= n * m else (n - 1) * -(-m // 256)
        assert int(torch.count_nonzero(x[:cut].view(torch.uint8))) == 0
