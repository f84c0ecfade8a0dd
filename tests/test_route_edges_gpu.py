"""Scored routing on the GPU at the edges of its contract, against the oracle in fp64.  Tolerances as in test_training_ops_gpu."""
import math

import numpy as np
import pytest
import torch

import paper_2506_14435_amd as M
from oracle import mote_oracle as O
from tests.test_training_ops_gpu import _check_route, _np, _router

pytestmark = pytest.mark.gpu


# one workgroup partly filled, a last one, shares of the channels; rows of the router that end inside a load of 1 KB
@pytest.mark.parametrize("T,d,E", [(1, 128, 1), (1, 2048, 16), (7, 256, 3), (33, 640, 60), (1, 8192, 64), (40, 4096, 33), (1055, 256, 40)])
def test_route_of_operands_among_other_data(T, d, E):
    """What lies around x and w_router has no part in the result."""
    g, x, w = _router(T, d, E, T + d + E)
    k = min(E, 4)
    outs = []
    for fill in (0.0, math.nan, 3e38):
        room = torch.full(((T + 40) * d + (d + 16) * E,), fill, dtype=torch.bfloat16, device="cuda")
        xs = room[4 * d:(4 + T) * d].view(T, d)
        ws = room[(T + 40) * d + 8 * E:(T + 40) * d + (8 + d) * E].view(d, E)
        xs.copy_(x)
        ws.copy_(w)
        r = M.mote_route(xs, ws, M.MoteRouting(k, renormalise=True), want_logits=True, want_stats=True)
        torch.cuda.synchronize()
        outs.append(r)
    for r in outs[1:]:
        for a, b in zip(outs[0], r):
            assert torch.equal(a, b)
    ref = O.route(_np(x), _np(w), k, renormalise=True)
    assert np.array_equal(outs[0].topk_idx.cpu().numpy(), ref["idx"])
