"""CPU checks of scored routing at the edges of its contract: what can be seen in the source, sizes, and argument checks that end
before a launch."""
import ctypes
import os
import re

import pytest

import paper_2506_14435_amd as M


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(M.LIB_PATH):
        from paper_2506_14435_amd import build
        build.build()
    return M.load_library()


def test_range_checked_loads_carry_their_whole_offset_in_the_lane():
    """route.hip reads tokens behind the last one as zeros through the range check of a buffer load, in which a scalar offset has
    no part: with the row of a token in it, a batch of one token read up to 31 rows behind x."""
    src = open(os.path.join(os.path.dirname(M.LIB_PATH), "csrc", "route.hip")).read()
    loads = re.findall(r"raw_buffer_load_b128\((.*?)\);", src)
    assert len(loads) == 2
    for args in loads:
        assert args.endswith(", 0, 0"), args


@pytest.mark.parametrize("d,E", [(256, 8), (2048, 64), (3584, 9), (3584, 64), (7168, 64), (8192, 33), (16384, 64), (65536, 64)])
def test_a_route_workspace_serves_every_smaller_batch(lib, d, E):
    """One buffer for the largest batch: sizes never fall, and what a size is made of for a smaller batch fits."""
    for f in (lib.mote_route_workspace_bytes, lib.mote_route_lean_workspace_bytes):
        counts = sorted({*range(0, 1100), *range(1100, 9000, 97), 16301, 1 << 20})
        sizes = [f(T, d, E) for T in counts]
        assert sizes == sorted(sizes)
    assert all(lib.mote_route_lean_workspace_bytes(T, d, E) <= lib.mote_route_workspace_bytes(T, d, E) for T in (0, 1, 64, 65, 1024, 1025))
    assert lib.mote_route_lean_workspace_bytes(0, d, E) == 0
    for T, dd, e in ((-1, d, E), (1 << 24, d, E), (4, 100, E), (4, d, 65)):
        assert lib.mote_route_lean_workspace_bytes(T, dd, e) == 0


def test_the_binding_asks_the_library_for_a_route_workspace(lib):
    """No rule of the library's is kept a second time in binding.py."""
    src = open(os.path.join(os.path.dirname(M.LIB_PATH), "binding.py")).read()
    body = src[src.index("def mote_route("):src.index("def mote_route_backward(")]
    assert "64" not in body and "1 << 17" not in body
    assert lib.mote_route_lean_workspace_bytes(1, 2048, 16) == 0 < lib.mote_route_lean_workspace_bytes(1, 3584, 64)


def _call(lib, T, d, E, ws, ws_bytes, counts=None):
    cfg = ctypes.byref(M.binding.MoteRoutingStruct(0, 2, 1, 1, 1, 0, 1.0))
    return lib.mote_route(cfg, 256, 256, None, None, T, d, E, 256, 256, None, counts, None, ws, ws_bytes, None)


def test_route_workspace_below_the_least_is_refused(lib):
    """Refusals only, before any launch: neither room for a split nor for the weights laid out."""
    for T, d, E in ((65, 256, 8), (512, 3584, 64), (1025, 2048, 64)):
        assert _call(lib, T, d, E, 256, 512) == 3 and _call(lib, T, d, E, None, 1 << 30) == 1 and _call(lib, T, d, E, 128, 1 << 30) == 1
        assert _call(lib, T, d, E, 256, 1024, counts=256) == 3
    assert _call(lib, 4, 256, 8, 256, 16, counts=256) == 3


def test_sizes_of_a_description_do_not_part_from_what_the_kernels_write():
    """Outputs are allocated by top_k and d, kernels write by the struct and read the parameters: neither can be set on its own."""
    r, block = M.MoteRouting(2), M.MoteResidual(256)
    assert r.top_k == 2 and block.d == 256
    for obj, name in ((r, "top_k"), (block, "d")):
        with pytest.raises(AttributeError):
            setattr(obj, name, 4)
    r.struct.top_k = 3
    assert r.top_k == 3
