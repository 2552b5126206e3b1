"""How much a gradient slot takes: counted before anything is made of it, and checked against the launches."""

import ctypes as C
import os
import subprocess
import sys

import pytest

from paper_2306_08881_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILES = (1 << 22) - 1  # of a kind, at most


def ask(shapes, bits, ranks):
    """(status, bytes) of acp_adamw_grads_bytes for gradients of these ranks at made-up addresses."""
    lib = L.load()
    opt = C.c_void_p()
    flat = [d for s in shapes for d in s]
    assert lib.acp_adamw_init(C.byref(opt), len(shapes), (C.c_int32 * len(shapes))(*[len(s) for s in shapes]),
                              (C.c_int64 * len(flat))(*flat), bits, None, 0) == L.ACP_OK
    grads = (L.AdamwGrad * len(shapes))(*[L.AdamwGrad(None, 256, 256, 0, r) if r else L.AdamwGrad(256, None, None, 0, 0)
                                          for r in ranks])
    size = C.c_int64()
    status = lib.acp_adamw_grads_bytes(opt, grads, C.byref(size))
    lib.acp_adamw_destroy(opt)
    return status, size.value


@pytest.mark.parametrize("shape,bits,rank,more", [
    ((2048 * TILES,), 32, 0, (2048 * TILES + 4,)),  # (a tile of less than a word is of another kind)
    ((16 * 256 * TILES,), 8, 0, (16 * 256 * TILES + 1,)),
    ((16 * TILES, 1), 8, 0, None),                        # 256 rows a block: far from the limit
    ((64 * TILES, 4), 32, 2, (64 * TILES + 1, 4)),        # narrow: the one block of 64 rows
    ((16 * TILES, 255), 8, 2, (16 * TILES + 1, 255)),     # narrow: blocks of 16 rows
    ((16 * TILES, 256), 32, 4, (16 * TILES + 1, 256)),    # one group of rows a tile
    ((16 * TILES, 256), 8, 4, None),                      # four
    ((256 * (TILES - 1), 1), 32, 1, (256 * (TILES - 1) + 1, 1)),  # Gram slices of A, and one of B
], ids=str)
def test_tiles_of_a_kind(shape, bits, rank, more):
    status, size = ask([shape], bits, [rank])
    assert status == L.ACP_OK and size > 0
    if more:
        assert ask([more], bits, [rank])[0] == L.ACP_E_INVALID


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shape", [(4, 1 << 38), (1 << 32, 256), (1 << 38, 4)], ids=str)
def test_refused_without_memory(shape, bits):
    """What init takes at most is refused by a process that may take no more than 256 MiB for it (the lists of
    its tiles would be 8 to 64 GiB)."""
    code = f"""
import ctypes as C, resource, sys
sys.path.insert(0, {ROOT!r}); sys.path.insert(0, {os.path.join(ROOT, "tests")!r})
import test_adamw_limits_host as T
T.ask([(3, 3)], {bits}, [0])
pages = int(open("/proc/self/statm").read().split()[0])
limit = pages * resource.getpagesize() + (256 << 20)
resource.setrlimit(resource.RLIMIT_AS, (limit, limit))
print("status", T.ask([{shape!r}], {bits}, [0])[0])
"""
    p = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert f"status {L.ACP_E_INVALID}" in p.stdout, p.stdout + p.stderr


@pytest.mark.parametrize("rank,ok", [(128, True), (129, False)])
def test_threads_of_a_launch(rank, ok):
    """Narrow tiles go with the products' launch, whose workgroups have 512 threads above rank 128: together
    they pass 2^32 there, though neither kind of tile does."""
    rows = 16 * TILES
    status, _ = ask([(rows, 250), (rows, 256)], 32, [rank, rank])
    assert status == (L.ACP_OK if ok else L.ACP_E_INVALID)
