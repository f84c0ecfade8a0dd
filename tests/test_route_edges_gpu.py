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


def _two_of_different_scores(T, d, E, seed, groups):
    """Tokens that are one token but for a channel that only the other experts see: experts a and b have quite different scores and
    a bias that brings their keys (with groups: the scores of their groups) together, so that the rows' denominators order them."""
    g, x, w = _router(1, d, E, seed)
    x[0, torch.randperm(d - 1, generator=g)[:4]] *= 20.0
    w = (w.float() * 0.3).to(torch.bfloat16)
    x = x.expand(T, d).clone()
    x[:, d - 1] = (torch.randn(T, generator=g) * 2.0 ** -22).to(torch.bfloat16)
    x[0, d - 1] = 0.0
    w[d - 1] = torch.randn(E, generator=g).to(torch.bfloat16)
    logits = _np(x[:1]) @ _np(w)
    s = np.exp(logits[0] - logits[0].max())
    s /= s.sum()
    bias = torch.zeros(E)
    if groups == 1:
        a, b = np.argsort(-s)[[0, 12]]
        w[d - 1, [a, b]] = 0.0
        bias[b] = float(s[a] - s[b])
    else:
        n = E // groups
        top2 = np.sort(s.reshape(groups, n), axis=1)[:, -2:].sum(axis=1)
        ga, gb = np.argsort(-top2)[[0, groups // 2]]
        w[d - 1, n * ga:n * ga + n] = 0.0
        w[d - 1, n * gb:n * gb + n] = 0.0
        best = n * gb + np.argmax(s[n * gb:n * gb + n])
        bias[best] = float(top2[ga] - top2[gb])                        # the two groups' scores meet
    return x, w, bias


@pytest.mark.parametrize("T", [32, 1056])                              # the kernel of few tokens and that of many
@pytest.mark.parametrize("groups,k", [(1, 1), (1, 4), (8, 4)])
def test_route_orders_keys_that_hang_on_the_denominator(T, groups, k):
    """Softmax scores with a bias: the key of an expert whose own logit is settled still moves with the other experts' logits."""
    cfg = dict(n_groups=groups, top_groups=1, group_top=2) if groups > 1 else {}
    flips = 0
    for seed in range(6):
        x, w, bias = _two_of_different_scores(T, 2048, 64, seed, groups)
        ref, _ = _check_route(x, w, bias, None, k, **cfg)
        flips += len(np.unique(ref["idx"][:, 0])) > 1
    assert flips >= 3                                                  # tokens of one batch fall on either side


@pytest.mark.parametrize("T", [64, 1056])
@pytest.mark.parametrize("E,groups", [(8, 4), (48, 6)])
@pytest.mark.parametrize("size", [1e2, 1e3, 1e4, 1e6])
def test_route_groups_whose_keys_cancel(T, E, groups, size):
    """A group's score of a large key and one as large below zero: what its fp32 sum has lost is of the keys' size, not of the sum's."""
    g, x, w = _router(T, 256, E, int(size) + E)
    n = E // groups
    bias = torch.zeros(E)
    bias[0::n] = size * (1 + torch.rand(groups, generator=g))
    bias[1::n] = -bias[0::n]
    for i in range(2, n):                                              # of more than two, the others are below
        bias[i::n] = -4 * size
    for score in ("softmax", "sigmoid"):
        ref, _ = _check_route(x, w, bias, None, 4, score=score, n_groups=groups, top_groups=2, group_top=2)
        assert len(np.unique(ref["idx"] // n)) == groups               # no group is always in
