"""Python binding of the library's AdamW operators (argument marshalling only).

``AdamW`` owns one ``acp_adamw``, the device block of its moments and a gradient block per slot (torch
uint8 tensors); its methods carry the C names without the ``acp_adamw_`` prefix and pass torch device
pointers and the current HIP stream through.

The optimiser's own memory comes from the stream of the call that makes it (``bind``, ``set_grads``, which
wait for that stream), and stays until what other streams were given on it has ended.  Work on several streams
is put in order by the caller; a stream that the caller made by other means than torch outlives the optimiser.
"""

from __future__ import annotations

import ctypes as C
from typing import Dict, Optional, Sequence, Tuple

import torch

from . import _lib as L

# the current stream's address without a Stream object, which takes half as long as a small step
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _ptr(t, dtypes, numel: int, what: str, device) -> int:
    if t.dtype not in dtypes or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous device tensor of {' or '.join(str(d) for d in dtypes)}")
    if t.device != device:
        raise ValueError(f"{what}: expected a tensor on {device}, got one on {t.device}")
    if t.numel() != numel:
        raise ValueError(f"{what}: expected {numel} elements, got {t.numel()}")
    return t.data_ptr()


class AdamW:
    """AdamW over many tensors at once (see include/acp.h).

    ``shapes``: the parameters' shapes; ``params``: their fp32 device tensors, one per shape, updated in
    place (None: norms only); ``copies``: bfloat16 tensors written beside them (None, or None for some);
    ``bits``: 32 or 8 per value of the moments; ``decay``: whether weight decay applies, per tensor (all);
    ``seed``: of the rounding of 8-bit moments.
    """

    def __init__(self, shapes: Sequence[Sequence[int]], params: Optional[Sequence] = None,
                 copies: Optional[Sequence] = None, *, bits: int = 32, decay: Optional[Sequence[bool]] = None,
                 seed: int = 0, device=None, stream=None):
        self.opt = None
        self.lib = L.load()
        self.shapes = [tuple(int(d) for d in s) for s in shapes]
        self.bits, self.seed = bits, seed
        count = len(self.shapes)
        self.numels = []
        for s in self.shapes:
            k = 1
            for d in s:
                k *= d
            self.numels.append(k)
        ndims = (C.c_int32 * count)(*[len(s) for s in self.shapes])
        flat = [d for s in self.shapes for d in s]
        dims = (C.c_int64 * len(flat))(*flat)
        no_decay = None
        if decay is not None:
            if len(decay) != count:
                raise ValueError(f"expected {count} decay flags, got {len(decay)}")
            no_decay = (C.c_uint8 * count)(*[0 if d else 1 for d in decay])
        opt = C.c_void_p()
        st = self.lib.acp_adamw_init(C.byref(opt), count, ndims, dims, bits, no_decay, seed)
        if st != L.ACP_OK:
            raise L.AcpError(st, "acp_adamw_init")
        self.opt = opt
        self.state, self.clip = None, None
        self.params, self.copies = None, None
        self._grads: Dict[int, tuple] = {}
        self._streams: Dict[int, object] = {}  # that calls were made on, by address
        self.bind(params, copies, device, stream)

    def _check(self, status: int, where: str):
        if status != L.ACP_OK:
            raise L.AcpError(status, where, self.lib.acp_adamw_last_error(self.opt).decode())

    def _stream(self, stream) -> int:
        s = _current_stream(self.device.index) if stream is None else stream.cuda_stream
        if s not in self._streams and self.state is not None:
            self._streams[s] = torch.cuda.current_stream(self.device) if stream is None else stream
            self._record(self.state, self.clip, *(block for _, block in self._grads.values()))
        return s

    def _record(self, *tensors):
        """The memory of these is not given to others before what the streams have on it has ended."""
        for t in tensors:
            for s in self._streams.values():
                t.record_stream(s)

    def _clip(self, clip) -> int:
        return self._clip_ptr if clip is self.clip else _ptr(clip, (torch.float32,), 2, "clip", self.device)

    # ---- setup
    def state_bytes(self) -> int:
        v = C.c_int64()
        self._check(self.lib.acp_adamw_state_bytes(self.opt, C.byref(v)), "acp_adamw_state_bytes")
        return v.value

    def bind(self, params=None, copies=None, device=None, stream=None):
        """A new state block with zero moments; gradients have to be set again."""
        if device is None:
            device = next((t.device for t in params or () if t is not None), "cuda")
        device = torch.device(device)
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())

        def addresses(ts, dtype, what):
            if ts is None:
                return None
            if len(ts) != len(self.shapes):
                raise ValueError(f"expected {len(self.shapes)} {what}s, got {len(ts)}")
            return (C.c_void_p * len(ts))(*[None if t is None else _ptr(t, (dtype,), k, what, device)
                                            for t, k in zip(ts, self.numels)])

        p, c = addresses(params, torch.float32, "parameter"), addresses(copies, torch.bfloat16, "copy")
        on = torch.cuda.current_stream(device) if stream is None else stream
        with torch.cuda.stream(on), torch.cuda.device(device):
            nbytes = self.state_bytes()
            clip = torch.zeros(2, device=device)
            state = torch.empty(nbytes, dtype=torch.uint8, device=device)
            self._check(self.lib.acp_adamw_bind(self.opt, state.data_ptr(), nbytes, p, c, on.cuda_stream),
                        "acp_adamw_bind")
        self.device, self._streams = device, {}
        self.clip, self._clip_ptr = clip, clip.data_ptr()
        self.state, self.params, self.copies = state, params, copies
        self._grads = {}

    def moments(self) -> Dict[str, object]:
        """Views of the state: flat "m" and "v" (fp32), or with 8 bits "m" and "v" (float8_e4m3fn, of m and
        sqrt(v)) and the scales of their blocks, "m_scale" and "v_scale"."""
        v = [C.c_int64() for _ in range(6)]
        self._check(self.lib.acp_adamw_regions(self.opt, *[C.byref(x) for x in v]), "acp_adamw_regions")
        elems, blocks, *offs = (x.value for x in v)
        if self.bits == 32:
            return {k: self.state[o:o + 4 * elems].view(torch.float32) for k, o in zip(("m", "v"), offs)}
        views = {k: self.state[o:o + elems].view(torch.float8_e4m3fn) for k, o in zip(("m", "v"), offs)}
        views.update({k: self.state[o:o + 4 * blocks].view(torch.float32)
                      for k, o in zip(("m_scale", "v_scale"), offs[2:])})
        return views

    def tensor_info(self, tensor: int) -> Tuple[int, int, int, int, int]:
        """(first element, first block, blocks, rows of a block, columns of a block) of a tensor."""
        a = [C.c_int64() for _ in range(3)]
        b = [C.c_int32() for _ in range(2)]
        self._check(self.lib.acp_adamw_tensor_info(self.opt, tensor, *[C.byref(x) for x in a + b]),
                    "acp_adamw_tensor_info")
        return tuple(x.value for x in a + b)

    def set_grads(self, grads: Sequence, slot: int = 0, stream=None):
        """Gradients of a slot, one entry per tensor: a tensor (fp32 or bfloat16), or a pair of fp32 factors
        (a, b) of the gradient a b^T.  They are kept, and read by every later call that names the slot."""
        if len(grads) != len(self.shapes):
            raise ValueError(f"expected {len(self.shapes)} gradients, got {len(grads)}")
        arr = (L.AdamwGrad * len(grads))()
        for g, shape, numel, x in zip(grads, self.shapes, self.numels, arr):
            if isinstance(g, (tuple, list)):
                a, b = g
                if a.dim() != 2 or b.dim() != 2 or a.shape[1] != b.shape[1] or a.shape[1] == 0:
                    raise ValueError("factors are matrices with one column per rank")
                n = shape[0] if len(shape) > 1 else 1
                x.rank = a.shape[1]
                x.a = _ptr(a, (torch.float32,), n * x.rank, "factor", self.device)
                x.b = _ptr(b, (torch.float32,), numel // n * x.rank, "factor", self.device)
            else:
                x.grad = _ptr(g, (torch.float32, torch.bfloat16), numel, "gradient", self.device)
                x.type = L.ACP_GRAD_BF16 if g.dtype == torch.bfloat16 else L.ACP_GRAD_FP32
        v = C.c_int64()
        self._check(self.lib.acp_adamw_grads_bytes(self.opt, arr, C.byref(v)), "acp_adamw_grads_bytes")
        on = torch.cuda.current_stream(self.device) if stream is None else stream
        with torch.cuda.stream(on), torch.cuda.device(self.device):
            block = torch.empty(v.value, dtype=torch.uint8, device=self.device)
            self._check(self.lib.acp_adamw_set_grads(self.opt, slot, arr, block.data_ptr(), v.value, on.cuda_stream),
                        "acp_adamw_set_grads")
        self._record(block)
        self._grads[slot] = (list(grads), block)

    # ---- the step
    def norm(self, max_norm: float = float("inf"), scale: float = 1.0, slot: int = 0, clip=None, stream=None):
        """The gradients' norm and clip coefficient, into ``clip`` (two floats on the device; by default one
        the optimiser keeps), which is returned and can be handed to ``step``."""
        clip = self.clip if clip is None else clip
        self._check(self.lib.acp_adamw_norm(self.opt, slot, scale, max_norm, self._clip(clip), self._stream(stream)),
                    "acp_adamw_norm")
        return clip

    def step(self, step: int, lr: float, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
             weight_decay: float = 0.01, scale: float = 1.0, clip=None, slot: int = 0, stream=None):
        """Step ``step`` (from 1) with a slot's gradients, times ``scale`` and the coefficient of ``clip``."""
        h = L.AdamwHyper(lr, betas[0], betas[1], eps, weight_decay, scale)
        c = None if clip is None else self._clip(clip)
        self._check(self.lib.acp_adamw_step(self.opt, slot, step, C.byref(h), c, self._stream(stream)), "acp_adamw_step")

    def close(self):
        if getattr(self, "opt", None):
            self.lib.acp_adamw_destroy(self.opt)
            self.opt = None
        self.state, self._grads = None, {}

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
