"""The AdamW binding's checks of tensors, on stand-ins for tensors of two GPUs."""

import pytest
import torch

from paper_2306_08881_amd import adamw

HERE, THERE = torch.device("cuda", 0), torch.device("cuda", 1)


class Tensor:
    """What the binding asks of a tensor."""

    is_cuda = True

    def __init__(self, device, *shape, dtype=torch.float32):
        self.device, self.shape, self.dtype = device, shape, dtype

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def numel(self):
        return torch.Size(self.shape).numel()

    def data_ptr(self):
        return 4096


@pytest.fixture
def opt():
    """An optimiser of one 6 x 8 tensor on the first GPU, without a library: a call to it would fail."""
    x = object.__new__(adamw.AdamW)
    x.opt = x.lib = x.clip = x.state = None
    x.shapes, x.numels, x.device = [(6, 8)], [48], HERE
    x._grads, x._streams = {}, {}
    return x


def test_gradients_of_another_device(opt):
    for bad in (Tensor(THERE, 6, 8), Tensor(THERE, 6, 8, dtype=torch.bfloat16), (Tensor(THERE, 6, 2), Tensor(HERE, 8, 2)),
                (Tensor(HERE, 6, 2), Tensor(THERE, 8, 2))):
        with pytest.raises(ValueError, match="cuda:0, got one on cuda:1"):
            opt.set_grads([bad])


def test_parameters_of_another_device(opt):
    opt.shapes, opt.numels = [(6, 8)] * 2, [48] * 2
    here, there = Tensor(HERE, 6, 8), Tensor(THERE, 6, 8)
    with pytest.raises(ValueError, match="parameter: .* cuda:1"):
        opt.bind([here, there])
    with pytest.raises(ValueError, match="parameter: .* cuda:1"):
        opt.bind([there, here], device=HERE)
    with pytest.raises(ValueError, match="copy: .* cuda:1"):
        opt.bind([here, here], [Tensor(HERE, 6, 8, dtype=torch.bfloat16), Tensor(THERE, 6, 8, dtype=torch.bfloat16)])
    assert opt.device == HERE  # a call that is refused leaves the optimiser where it was


def test_clip_of_another_device(opt):
    with pytest.raises(ValueError, match="clip: .* cuda:1"):
        opt._clip(Tensor(THERE, 2))
    assert opt._clip(Tensor(HERE, 2)) == 4096
