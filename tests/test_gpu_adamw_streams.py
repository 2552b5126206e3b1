"""AdamW on streams other than the current one: the optimiser's own memory is ready for them and stays theirs."""

import pytest

import adamw_ref as R

pytestmark = pytest.mark.gpu

SHAPES = [(1000, 700), (33, 1021), (700,), (40, 2)]


def tensors(seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    p = [torch.randn(s, generator=gen, device="cuda") for s in SHAPES]
    g = [torch.randn(s, generator=gen, device="cuda") * 1e-2 for s in SHAPES]
    return p, g


def keep_busy(x):
    """Some tenths of a second of work on the current stream."""
    for _ in range(400):
        x = x @ x
    return x


@pytest.mark.parametrize("bits", [32, 8])
def test_stream_argument(bits):
    """Bound, given gradients and stepped on a side stream, behind whose back the current stream still has
    writes to memory that it has given back, of the sizes that the optimiser asks for."""
    import torch
    from paper_2306_08881_amd.adamw import AdamW
    p, g = tensors(1)
    opt = AdamW(SHAPES, p, bits=bits, seed=3)
    opt.set_grads(g)
    opt.step(1, clip=opt.norm(0.1), **R.HYPER)
    sizes = [opt.state.numel(), opt._grads[0][1].numel(), 2 * 4]
    want = [x.clone() for x in p] + [x.clone() for x in opt.moments().values()] + [opt.clip.clone()]
    opt.close()
    q, g = tensors(1)
    side = torch.cuda.Stream()
    x = torch.eye(8192, dtype=torch.bfloat16, device="cuda")
    keep_busy(x)  # (the library is loaded)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    old = [torch.empty(k, dtype=torch.uint8, device="cuda") for k in sizes]
    y = keep_busy(x)
    for o in old:
        o.fill_(0xFF)
    del old, o
    opt = AdamW(SHAPES, q, bits=bits, seed=3, stream=side)
    opt.set_grads(g, stream=side)
    clip = opt.norm(0.1, stream=side)
    opt.step(1, clip=clip, stream=side, **R.HYPER)
    torch.cuda.synchronize()
    got = q + list(opt.moments().values()) + [clip]
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(want, got))
    assert float(y[0, 0]) == 1.0


@pytest.mark.parametrize("by", ["argument", "context"])
def test_memory_stays_for_other_streams(by):
    """Blocks that a call on a side stream still reads are not handed out again when the optimiser has given
    them up: a slot set again, a state bound again."""
    import torch
    from paper_2306_08881_amd.adamw import AdamW
    p, g = tensors(2)
    opt = AdamW(SHAPES, p)
    opt.set_grads(g)
    want, _ = tensors(2)
    ref = AdamW(SHAPES, want)
    ref.set_grads(g)
    ref.step(1, **R.HYPER)
    side = torch.cuda.Stream()
    x = torch.eye(8192, dtype=torch.bfloat16, device="cuda")
    keep_busy(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.record_stream(side)
        keep_busy(x)
        if by == "context":
            opt.step(1, **R.HYPER)
    if by == "argument":
        opt.step(1, stream=side, **R.HYPER)
    gone = [(opt._grads[0][1].data_ptr(), opt._grads[0][1].numel()), (opt.state.data_ptr(), opt.state.numel())]
    opt.set_grads(g)
    opt.close()
    for at, size in gone:
        new = torch.empty(size, dtype=torch.uint8, device="cuda")
        assert side.query() or not (new.data_ptr() < at + size and at < new.data_ptr() + size)
        new.fill_(0xFF)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, p))
