"""The training-step operators on the GPU against the oracle in fp64.

Tolerances, all per element: a result rounded once to type t is off by half a step, finfo(t).eps / 2 of its value.  What is
computed in fp32 on the way is off by a number of roundings (u = 2^-24 each) of the *magnitude* of the expression: the same
sums and products over absolute values.  The number is counted generously: 64 for a chain of a few operations and sums by a
tree, and the number of terms for sums one after the other."""
import math

import numpy as np
import pytest
import torch

import paper_2506_14435_amd as M
import workloads as W
from oracle import mote_oracle as O
from tests.mote_testlib import GpuProblem

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
TINY = 1e-37                                 # below the smallest normal fp32 value and bf16 value, times a few


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _close(got, want, tol, what):
    got = _np(got)
    assert got.shape == want.shape, what
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


# -------------------------------------------------------------------------------------------------------- routing
def _router(T, d, E, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16)
    w = (torch.randn(d, E, generator=g) * d ** -0.5).to(torch.bfloat16)
    return g, x, w


def _same_selection(got, ref, x, w, bias):
    """The oracle's indices, but that two experts may be in either order where fp64 itself does not tell them apart.  A sum of d
    products rounded in any order is off by at most d 2^-53 sum |x w| = e; a score (at most 1) of it by 2 e and the three
    roundings, each below 2^-52, of exp, the sum of the row and the quotient.  Two such keys differ by at most twice that.
    Equal columns with equal bias have equal keys however they are rounded: the lower index, always."""
    xd, wd = np.abs(_np(x)), np.abs(_np(w))
    for t, j in np.argwhere(got != ref["idx"]):
        a, b = got[t, j], ref["idx"][t, j]
        assert a >= 0 and b >= 0, (t, j)
        e = x.shape[1] * 2.0 ** -53 * max(xd[t] @ wd[:, a], xd[t] @ wd[:, b])
        assert abs(ref["keys"][t, a] - ref["keys"][t, b]) <= 2 * (2 * e + 3 * 2.0 ** -52), (t, j, a, b)
        assert not torch.equal(w[:, a], w[:, b]) or (bias is not None and bias[a] != bias[b]), (t, j, a, b)
    swapped = (got != ref["idx"]).any(axis=1)
    assert np.array_equal(np.sort(got[swapped], axis=1), np.sort(ref["idx"][swapped], axis=1)) or swapped.sum() <= 2 + len(got) // 100
    return ~swapped


def _check_route(x, w, bias, mask, k, **cfg):
    """Runs mote_route with everything it can return and compares; returns the oracle's dict."""
    T, E = x.shape[0], w.shape[1]
    xd, wd = _np(x), _np(w)
    names = dict(cfg)
    ref = O.route(xd, wd, k, select_bias=None if bias is None else bias.numpy(), token_mask=None if mask is None else mask.numpy(), **names)
    routing = M.MoteRouting(k, **cfg)
    dev = lambda t: None if t is None else t.cuda()
    got = M.mote_route(dev(x), dev(w), routing, select_bias=dev(bias), token_mask=dev(mask), want_logits=True, want_stats=True)
    lean = M.mote_route(dev(x), dev(w), routing, select_bias=dev(bias), token_mask=dev(mask))
    torch.cuda.synchronize()
    same = _same_selection(got.topk_idx.cpu().numpy(), ref, x, w, bias)
    assert torch.equal(got.topk_idx, lean.topk_idx) and torch.equal(got.topk_w.isnan(), lean.topk_w.isnan())
    assert torch.equal(got.topk_w.nan_to_num(), lean.topk_w.nan_to_num()) and lean.logits is None and lean.counts is None
    counts = got.topk_idx.cpu().numpy()
    assert np.array_equal(got.counts.cpu().numpy(), np.bincount(counts[counts >= 0], minlength=E))
    # logits: rounded once, sums off by at most 2^-20 of the magnitude; scores follow an error d of the logits by exp(2 d)
    with np.errstate(invalid="ignore", over="ignore"):
        err_l = U * np.abs(ref["logits"]) + 2.0 ** -20 * (np.abs(xd) @ np.abs(wd)) + TINY
        spread = np.abs(ref["logits"]).max(axis=1, initial=0.0) * 2
        finite = np.isfinite(ref["logits"]).all(axis=1) & np.isfinite(err_l).all(axis=1) & (np.abs(ref["logits"]) < 3e38).all(axis=1)
        rel = 2 * err_l.max(axis=1, initial=0.0) + U * (64 + 2 * spread)
        finite &= same
    _close(got.logits[torch.from_numpy(finite)], ref["logits"][finite], err_l[finite], "logits")
    _close(got.topk_w[torch.from_numpy(finite)], ref["w"][finite], rel[finite, None] * np.abs(ref["w"][finite]) + TINY, "weights")
    if (finite | ~same).all():
        live = np.ones(T, bool) if mask is None else mask.numpy() != 0
        _close(got.score_sum, ref["score_sum"], (rel[live, None] * ref["scores"][live]).sum(axis=0) + U * ref["score_sum"] + TINY, "score sums")
    return ref, got


@pytest.mark.parametrize("T,d,E,k", [(1, 128, 1, 1), (1, 2048, 16, 2), (3, 256, 2, 2), (5, 896, 8, 2), (31, 384, 7, 3), (33, 128, 33, 8), (64, 3584, 64, 8),
                                     (65, 256, 60, 4), (130, 640, 17, 5), (257, 1536, 48, 6), (1025, 2048, 64, 6), (2, 4096, 64, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_shapes(T, d, E, k, score):
    g, x, w = _router(T, d, E, T + d + E)
    bias = torch.randn(E, generator=g) * 0.05
    _check_route(x, w, None, None, k, score=score)
    _check_route(x, w, bias, None, k, score=score, renormalise=True, scale=2.5)
    if T > 1:
        mask = (torch.rand(T, generator=g) < 0.7).to(torch.uint8)
        _check_route(x, w, bias, mask, k, score=score, renormalise=True)


@pytest.mark.parametrize("E,G,top,gt,k", [(8, 4, 2, 1, 2), (8, 4, 2, 2, 4), (64, 8, 4, 2, 8), (60, 6, 3, 1, 4), (64, 32, 5, 2, 8), (64, 64, 8, 1, 8),
                                          (12, 1, 1, 2, 3), (9, 3, 3, 2, 8), (34, 17, 2, 2, 4), (63, 7, 1, 2, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_groups(E, G, top, gt, k, score):
    g, x, w = _router(150, 256, E, E * 31 + G)
    bias = torch.randn(E, generator=g) * 0.1
    for b in (None, bias):
        _check_route(x, w, b, None, k, score=score, n_groups=G, top_groups=top, group_top=gt, renormalise=True)


# few tokens, rows so wide that the channels go to several workgroups; d / 64 that the shares do not divide, odd E, more shares than waves
@pytest.mark.parametrize("T,d,E,k", [(1, 4096, 16, 2), (64, 2048, 33, 8), (17, 3456, 7, 3), (40, 8320, 64, 8), (33, 16384, 5, 2), (2, 65536, 64, 6)])
def test_route_of_wide_rows(T, d, E, k):
    g, x, w = _router(T, d, E, T + d + E)
    bias = torch.randn(E, generator=g) * 0.05
    mask = (torch.rand(T, generator=g) < 0.7).to(torch.uint8)
    _check_route(x, w, None, None, k)
    _check_route(x, w, bias, mask, k, score="sigmoid", renormalise=True)
    # pairs of columns that fp32 sums cannot tell apart, and one that is the same
    w[:, 1] = w[:, 0]
    w[:, 3] = w[:, 2]
    x[:, d - 1] = (torch.randn(T, generator=g) * 2.0 ** -20).to(torch.bfloat16)
    w[d - 1, 1] = 1.0
    cfg = dict(score="softmax", renormalise=True)
    _check_route(x, w, None, None, k, **cfg)
    # the call without memory for shares: the same experts
    args = (x.cuda(), w.cuda(), M.MoteRouting(k, **cfg))
    one, many = M.mote_route(*args, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), M.mote_route(*args)
    torch.cuda.synchronize()
    assert torch.equal(one.topk_idx, many.topk_idx) and torch.allclose(one.topk_w, many.topk_w, rtol=U * 200, atol=0)
    x[0, d // 2] = math.nan
    r = M.mote_route(x.cuda(), w.cuda(), M.MoteRouting(k), want_stats=True)
    torch.cuda.synchronize()
    assert ((r.topk_idx >= 0) & (r.topk_idx < E)).all() and r.topk_w[0].isnan().all() and not r.topk_w[1:].isnan().any()


@pytest.mark.parametrize("T,d,E,k", [(70, 7168, 64, 8), (200, 2048, 64, 6), (1024, 3584, 9, 2), (333, 2176, 35, 4)])
@pytest.mark.parametrize("split", [True, False])
def test_route_of_wide_rows_and_some_tokens(T, d, E, k, split):
    """Memory for shares of the channels or not: an equal pair of columns, a pair that fp32 sums cannot tell apart, a padded batch."""
    g, x, w = _router(T, d, E, T + d + E)
    w[:, 1] = w[:, 0]
    w[:, 3] = w[:, 2]
    x[:, d - 1] = (torch.randn(T, generator=g) * 2.0 ** -20).to(torch.bfloat16)
    w[d - 1, 1] = 1.0
    mask = (torch.rand(T, generator=g) < 0.7).to(torch.uint8)
    ref = O.route(_np(x), _np(w), k, token_mask=mask.numpy(), renormalise=True)
    need = M.load_library().mote_route_workspace_bytes(T, d, E)
    r = M.mote_route(x.cuda(), w.cuda(), M.MoteRouting(k, renormalise=True), token_mask=mask.cuda(), want_stats=True,
                     workspace=torch.empty(need if split else need - 256, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    same = _same_selection(r.topk_idx.cpu().numpy(), ref, x, w, None)
    # logits are off by e and rounded scores by 64 roundings: weights by exp(2 e)
    e = 2.0 ** -20 * (np.abs(_np(x)) @ np.abs(_np(w))).max(axis=1)
    _close(r.topk_w[torch.from_numpy(same)], ref["w"][same], (2 * e + 128 * U)[same, None] * ref["w"][same] + TINY, "weights")
    assert int(r.counts.sum()) == k * int(mask.sum())


# the kernel of many tokens, whose weights are laid out first
@pytest.mark.parametrize("E", [32, 64])
@pytest.mark.parametrize("gap", [2.0 ** -8, 2.0 ** -34])
def test_route_tells_close_logits_of_many_tokens_apart(gap, E):
    test_route_tells_close_logits_apart(gap, 1050, E)


@pytest.mark.parametrize("E", [6, 40])
def test_route_separates_three_and_more_of_many_tokens(E):
    test_route_separates_three_and_more(1040, E)


@pytest.mark.parametrize("E", [12, 44, 45])
def test_route_large_small_and_nonfinite_values_of_many_tokens(E):
    test_route_large_small_and_nonfinite_values(1033, E)


def test_route_agrees_with_the_plain_router():
    for T, d, E, k in ((64, 256, 4, 2), (300, 896, 8, 2), (2000, 2048, 16, 2), (100, 384, 40, 8)):
        _, x, w = _router(T, d, E, T)
        x, w = x.cuda(), w.cuda()
        idx, p, counts = M.mote_router_topk(x, w, k)
        r = M.mote_route(x, w, M.MoteRouting(k), want_stats=True)
        assert torch.equal(r.topk_idx, idx) and torch.equal(r.counts, counts)
        assert torch.allclose(r.topk_w, p, rtol=U * 200, atol=0)
        bal = M.mote_router_balance(x, w, k)
        assert torch.allclose(r.score_sum, bal[4], rtol=U * 200, atol=0)


def test_route_ties_go_to_the_lower_index():
    g, x, w = _router(97, 512, 24, 3)
    w[:, 13] = w[:, 2]                        # exact ties of whole columns, in and across groups
    w[:, 14] = w[:, 3]
    w[:, 20:24] = w[:, 4:8]
    for cfg in (dict(), dict(score="sigmoid"), dict(n_groups=6, top_groups=3, group_top=2), dict(score="sigmoid", n_groups=6, top_groups=2)):
        _check_route(x, w, None, None, 6, **cfg)
        _check_route(x, w, torch.zeros(24), None, 6, **cfg)
    _check_route(torch.zeros(5, 512, dtype=torch.bfloat16), w, None, None, 8)        # all logits zero
    _check_route(x, torch.zeros_like(w), None, None, 8, score="sigmoid", n_groups=4, top_groups=2, group_top=2)


# (T, E): the kernel of few tokens and that of many, with one and two tiles of experts
@pytest.mark.parametrize("T,E", [(20, 32), (200, 32), (200, 64), (33, 64)])
@pytest.mark.parametrize("gap", [2.0 ** -8, 2.0 ** -20, 2.0 ** -34])
def test_route_tells_close_logits_apart(gap, T, E):
    """Pairs of experts whose logits differ by gap times one product: far below an fp32 rounding of the sum, exact in fp64.
    Duplicated columns, one of which has one more small entry in a channel where x is small."""
    g, x, w = _router(T, 1024, E, 9)
    w[:, 1::2] = w[:, 0::2]
    x[:, 1023] = (torch.randn(T, generator=g) * gap).to(torch.bfloat16)
    w[1023, 0::2] = 0.0
    w[1023, 1::2] = (torch.randn(E // 2, generator=g)).to(torch.bfloat16)
    bias = (torch.randn(E // 2, generator=g) * 0.05).repeat_interleave(2)          # the same for both of a pair
    for b in (None, bias):
        for cfg in (dict(), dict(score="sigmoid", renormalise=True), dict(n_groups=16, top_groups=8, group_top=1),
                    dict(score="sigmoid", n_groups=8, top_groups=4, group_top=2), dict(n_groups=E // 2, top_groups=5, group_top=2)):
            _check_route(x, w, b, None, 8, **cfg)


@pytest.mark.parametrize("T,E", [(20, 6), (100, 6), (100, 40)])
def test_route_separates_three_and_more(T, E):
    """Three columns within a rounding of each other at the end of the selection, and all columns within one."""
    g, x, w = _router(T, 512, E, 29)
    w[:, 1] = w[:, 0]
    w[:, 2] = w[:, 0]
    x[:, 7] = (torch.randn(T, generator=g) * 2.0 ** -18).to(torch.bfloat16)
    w[7, 0:3] = torch.tensor([1.0, -1.0, 0.5]).to(torch.bfloat16)
    for k in (1, 2, 3, 4):
        _check_route(x, w, None, None, k)
        _check_route(x, w, torch.zeros(E), None, k, score="sigmoid")
    w[:, :] = w[:, :1]
    w[7] = torch.randn(E, generator=g).to(torch.bfloat16)
    _check_route(x, w, None, None, min(E, 8))
    _check_route(x, w, torch.zeros(E), None, min(E, 8), score="sigmoid", renormalise=True)


def test_route_switched_off_experts_and_empty_rows():
    g, x, w = _router(70, 256, 16, 11)
    for n_on in (16, 9, 3, 1, 0):
        bias = torch.zeros(16)
        bias[torch.randperm(16, generator=g)[n_on:]] = -math.inf
        for cfg in (dict(), dict(score="sigmoid", renormalise=True), dict(score="sigmoid", n_groups=4, top_groups=2, group_top=2, renormalise=True),
                    dict(n_groups=8, top_groups=5, group_top=1)):
            ref, got = _check_route(x, w, bias, None, 6, **cfg)
            assert torch.isfinite(got.topk_w).all()
    ref, got = _check_route(x, w, None, torch.zeros(70, dtype=torch.uint8), 4)        # nothing but padding
    assert (got.topk_idx == -1).all() and (got.topk_w == 0).all() and (got.score_sum == 0).all()
    _check_route(x, w, torch.full((16,), -3e38), None, 4, score="sigmoid")            # a mask of the lowest values is no mask
    _check_route(x, w, torch.tensor([math.inf] * 3 + [0.0] * 13), None, 4, score="sigmoid")


@pytest.mark.parametrize("T,E", [(40, 12), (90, 12), (90, 44), (90, 45)])
def test_route_large_small_and_nonfinite_values(T, E):
    g, x, w = _router(T, 256, E, 13)
    _check_route((x.float() * 300).to(torch.bfloat16), w, torch.randn(E, generator=g) * 0.01, None, 4, score="sigmoid", renormalise=True)   # saturated
    _check_route((x.float() * 300).to(torch.bfloat16), w, None, None, 4, score="softmax", renormalise=True)
    _check_route((x.float().abs() * -200).to(torch.bfloat16), w.abs(), None, None, 4, score="sigmoid", renormalise=True)      # all scores underflow fp32
    _check_route((x.float() * 1e30).to(torch.bfloat16), (w.float() * 1e20).to(torch.bfloat16), None, None, 4)                # logits beyond fp32
    _check_route((x.float() * 1e-30).to(torch.bfloat16), (w.float() * 1e-30).to(torch.bfloat16), None, None, 4)              # products below fp32
    _check_route((x.float() * 1e-38).to(torch.bfloat16), w, None, None, 4)                                                   # subnormal inputs
    bad = x.clone()
    bad[3, 5], bad[7, 0], bad[9, 1], bad[11, :] = math.nan, math.inf, -math.inf, math.nan
    for cfg in (dict(), dict(score="sigmoid", renormalise=True), dict(n_groups=E // 3 if E % 3 == 0 else 4, top_groups=2, group_top=2)):
        r = M.mote_route(bad.cuda(), w.cuda(), M.MoteRouting(4, **cfg), want_logits=True, want_stats=True)
        torch.cuda.synchronize()
        assert ((r.topk_idx >= -1) & (r.topk_idx < E)).all() and r.topk_w[[3, 11]].isnan().all()
        fine = [t for t in range(T) if t not in (3, 7, 9, 11)]
        ref = O.route(_np(x), _np(w), 4, **cfg)
        assert np.array_equal(r.topk_idx.cpu().numpy()[fine], ref["idx"][fine])
    bad_w = w.clone()                                     # a router column that is not a number: ranks last
    bad_w[5, 2] = math.nan
    r = M.mote_route(x.cuda(), bad_w.cuda(), M.MoteRouting(4, score="sigmoid"))
    ref = O.route(_np(x), np.delete(_np(w), 2, axis=1), 4, "sigmoid")["idx"]
    assert np.array_equal(r.topk_idx.cpu().numpy(), np.where(ref >= 2, ref + 1, ref))
    b = torch.zeros(E)
    b[4] = math.nan                                       # ranks last, is still chosen when nothing else is left
    b[5:] = -math.inf
    ref, got = _check_route(x, w, b, None, 6, score="sigmoid")
    assert (got.topk_idx[:, 4] == 4).all() and (got.topk_idx[:, 5] == -1).all()


def test_route_of_no_tokens():
    w = torch.zeros(256, 8, dtype=torch.bfloat16, device="cuda")
    r = M.mote_route(w.new_zeros(0, 256), w, M.MoteRouting(2), want_logits=True, want_stats=True)
    assert r.topk_idx.shape == (0, 2) and (r.counts == 0).all() and (r.score_sum == 0).all()
    dx, dw = M.mote_route_backward(w.new_zeros(0, 256), w, M.MoteRouting(2), r.logits, r.topk_idx, r.topk_w)
    assert dx.shape == (0, 256) and (dw == 0).all()


def _check_route_backward(x, w, idx, d_w, q, mask, score, renormalise, scale, logits=None):
    T, E = x.shape[0], w.shape[1]
    logits = (x.double() @ w.double()).float() if logits is None else logits
    g, dx, dw, mag = O.route_backward(_np(x), _np(w), _np(logits), idx.numpy(), _np(d_w), _np(q), None if mask is None else mask.numpy(), score,
                                      renormalise, scale)
    dev = lambda t: None if t is None else t.cuda()
    routing = M.MoteRouting(d_w.shape[1], score=score, renormalise=renormalise, scale=scale)
    got = M.mote_route_backward(dev(x), dev(w), routing, dev(logits), dev(idx), dev(d_w), dev(q), dev(mask))
    torch.cuda.synchronize()
    # dlogits: scores are off by U (64 + spread of the logits); then sums of E and T terms, three bf16 parts each
    spread = 2 * np.abs(_np(logits)).max(axis=1, initial=0.0, keepdims=True)
    per = U * (64 + 2 * spread) * mag
    _close(got[0], dx, (per + 3 * E * U * mag) @ np.abs(_np(w)).T + TINY, "dx")
    _close(got[1], dw, np.abs(_np(x)).T @ (per + (64 + 3 * T) * U * mag) + TINY, "dw")
    return got


@pytest.mark.parametrize("T,d,E,k", [(1, 128, 1, 1), (1, 2048, 16, 2), (3, 256, 2, 2), (31, 384, 7, 3), (33, 128, 33, 8), (64, 896, 64, 8), (65, 256, 60, 4),
                                     (257, 640, 17, 5), (1030, 512, 64, 8), (500, 1920, 8, 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_backward_shapes(T, d, E, k, score, renormalise):
    g, x, w = _router(T, d, E, T * 3 + d + E)
    idx = torch.from_numpy(O.route(_np(x), _np(w), k, score)["idx"])
    d_w, q = torch.randn(T, k, generator=g), torch.randn(E, generator=g) * 0.1
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8)
    _check_route_backward(x, w, idx, d_w, None, None, score, renormalise, 1.0)
    _check_route_backward(x, w, idx, d_w, q, mask, score, renormalise, 2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_backward_empty_repeated_and_padding(score, renormalise):
    g, x, w = _router(90, 256, 12, 17)
    idx = torch.randint(-1, 12, (90, 4), generator=g, dtype=torch.int32)       # -1 and the same expert twice
    idx[5], idx[6] = -1, 3
    d_w, q = torch.randn(90, 4, generator=g), torch.randn(12, generator=g)
    mask = torch.ones(90, dtype=torch.uint8)
    mask[40:] = 0
    dx, dw = _check_route_backward(x, w, idx, d_w, q, mask, score, renormalise, 0.7)
    assert (dx[40:] == 0).all()
    # rows behind the mask have no part, whatever they hold
    x2 = x.clone()
    logits = (x.double() @ w.double()).float()
    logits[40:] = math.nan
    d_w[40:] = math.inf
    idx[40:] = 1 << 20
    idx[3, 1] = 12                                                             # out of range: as -1
    idx_ref = idx.clone()
    idx_ref[3, 1] = -1
    idx_ref[40:] = -1
    r = M.MoteRouting(4, score=score, renormalise=renormalise, scale=0.7)
    a = M.mote_route_backward(x2.cuda(), w.cuda(), r, logits.cuda(), idx.cuda(), d_w.cuda(), q.cuda(), mask.cuda())
    logits[40:], d_w[40:] = 0.0, 0.0
    b = M.mote_route_backward(x2.cuda(), w.cuda(), r, logits.cuda(), idx_ref.cuda(), d_w.cuda(), q.cuda(), mask.cuda())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # one product asked for at a time gives the same bits
    only_dx = M.mote_route_backward(x2.cuda(), w.cuda(), r, logits.cuda(), idx_ref.cuda(), d_w.cuda(), q.cuda(), mask.cuda(), want_dw=False)
    only_dw = M.mote_route_backward(x2.cuda(), w.cuda(), r, logits.cuda(), idx_ref.cuda(), d_w.cuda(), q.cuda(), mask.cuda(), want_dx=False)
    assert only_dx[1] is None and torch.equal(only_dx[0], b[0]) and only_dw[0] is None and torch.equal(only_dw[1], b[1])


def test_route_backward_of_extreme_logits():
    g, x, w = _router(20, 128, 6, 19)
    logits = torch.randn(20, 6, generator=g) * 200                            # saturated and underflowing scores
    logits[4] = -300.0
    logits[5] = 300.0
    idx = torch.argsort(logits, dim=1, descending=True)[:, :3].to(torch.int32)
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            _check_route_backward(x, w, idx, torch.randn(20, 3, generator=g), torch.randn(6, generator=g), None, score, renormalise, 1.0, logits)


# --------------------------------------------------------------------------------------- the layer on a given routing
@pytest.mark.parametrize("cfg", [W.C1, W.C1.with_tokens(1, name="c1_T1"), W.decode_config(16, 8), W.MoteConfig("ragged", 384, 640, 8, 2, 211, seed=11),
                                 W.MoteConfig("many", 512, 1024, 16, 2, 3000, seed=12), W.MoteConfig("top1", 256, 512, 4, 1, 40, seed=3)],
                         ids=lambda c: c.name)
def test_layer_on_the_routers_own_routing_is_the_layer(cfg):
    gp = GpuProblem(cfg)
    names = ("topk_idx", "topk_p", "counts", "row_of", "q_x", "beta_x", "acc_gate", "acc_down", "out_f32")
    a, b = M.alloc_taps(gp.layer, cfg.n_tokens, names), M.alloc_taps(gp.layer, cfg.n_tokens, names)
    want = M.mote_layer_forward(gp.layer, gp.x, taps=a)
    got = M.mote_layer_forward_routed(gp.layer, gp.x, a["topk_idx"], a["topk_p"], taps=b)
    torch.cuda.synchronize()
    for n in names:
        assert torch.equal(a[n], b[n]), n
    assert torch.equal(got, want)


@pytest.mark.parametrize("T", [1, 30, 700])
def test_layer_skips_slots_without_an_expert(T):
    cfg = W.C1.with_tokens(T, name="holes")
    gp = GpuProblem(cfg)
    r = M.mote_route(gp.x, gp.w_router, M.MoteRouting(cfg.top_k, score="sigmoid", renormalise=True))
    idx, wt = r.topk_idx.clone(), r.topk_w.clone()
    idx[::3, 1] = -1
    idx[T // 2] = torch.tensor([1 << 30, -5], dtype=torch.int32)
    wt[T // 2] = math.nan                                                      # the weight of an empty slot is not read
    zero, safe = wt.clone(), idx.clone()
    gone = (idx < 0) | (idx >= cfg.n_experts)
    zero[gone], safe[gone] = 0.0, 2
    got = M.mote_layer_forward_routed(gp.layer, gp.x, idx, wt)
    want = M.mote_layer_forward_routed(gp.layer, gp.x, safe, zero)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.isfinite(got.float()).all()
    # one expert in both slots adds twice: the same sum as one slot with the weights together (one more fp32 rounding, bf16 output)
    idx, wt = torch.full_like(r.topk_idx, 1), torch.full_like(r.topk_w, 0.25)
    one = torch.tensor([1, -1], dtype=torch.int32, device="cuda").expand(T, 2).contiguous()
    twice, once = M.mote_layer_forward_routed(gp.layer, gp.x, idx, wt), M.mote_layer_forward_routed(gp.layer, gp.x, one, wt * 2)
    assert (twice.float() - once.float()).abs().max() <= 2.0 ** -7 * once.float().abs().max()


# ------------------------------------------------------------------------------------------------ residual and norms
def _block(d, post, pre, gated, g, a=0.75, b=0.5, eps=1e-6):
    """(MoteResidual, oracle's description)"""
    def vec(mean):
        return (mean + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16)

    dev, ora = {}, {}
    for n, kind in (("post", post), ("pre", pre)):
        gamma, beta = vec(1.0), vec(0.0)
        dev[n] = None if kind is None else M.MoteNorm(gamma.cuda(), beta.cuda() if kind == "layer" else None, eps)
        ora[n] = None if kind is None else (kind, _np(gamma), _np(beta), eps)
    gate = vec(0.5) if gated else None
    return (M.MoteResidual(d, post=dev["post"], gate=None if gate is None else gate.cuda(), pre=dev["pre"], residual_scale=a, branch_scale=b),
            dict(post=ora["post"], gate=_np(gate), pre=ora["pre"], residual_scale=a, branch_scale=b))


def _magnitudes(r, y, ora):
    """Magnitudes of z, total and normed, of the hats, and the rows' 1 / sqrt(var + eps)."""
    mean = lambda v: v.mean(axis=1, keepdims=True)
    z, _, inv_y = O._norm_parts(y, ora["post"])
    hat_y = z_mag = np.abs(y)
    if ora["post"] is not None:
        hat_y = inv_y * (np.abs(y) + mean(np.abs(y)))
        z_mag = hat_y * np.abs(ora["post"][1]) + (np.abs(ora["post"][2]) if ora["post"][0] == "layer" else 0.0)
    gate = 1.0 if ora["gate"] is None else np.abs(ora["gate"])
    total = O.residual_norm(r, y, **ora)[0]
    t_mag = abs(ora["residual_scale"]) * np.abs(r) + abs(ora["branch_scale"]) * gate * z_mag
    hat = n_mag = t_mag
    inv = np.ones_like(t_mag[:, :1])
    if ora["pre"] is not None:
        inv = O._norm_parts(total, ora["pre"])[2]
        grow = 1.0 + inv * np.sqrt(mean(t_mag ** 2))                     # an error of the row's values enters its scale too
        hat = inv * (t_mag + mean(t_mag)) * grow
        n_mag = hat * np.abs(ora["pre"][1]) + (np.abs(ora["pre"][2]) if ora["pre"][0] == "layer" else 0.0)
    return z_mag, t_mag, n_mag, hat_y, hat, inv_y, inv


SHAPES = [(1, 8), (1, 2048), (2, 128), (3, 896), (7, 520), (33, 1536), (5, 2056), (64, 3584), (9, 4096), (4, 8192), (3, 6008), (517, 264), (1200, 64)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("post,pre,gated", [("rms", "rms", True), ("layer", "layer", True), (None, "rms", False), ("rms", None, False),
                                            ("layer", "rms", False), (None, None, True)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_residual_norm_and_its_gradient(T, d, post, pre, gated, dt):
    g = torch.Generator().manual_seed(T * 10007 + d)
    block, ora = _block(d, post, pre, gated, g)
    r, y = (torch.randn(T, d, generator=g) * 2).to(dt), (torch.randn(T, d, generator=g) * 0.6 + 0.1).to(dt)
    d_total, d_normed = torch.randn(T, d, generator=g).to(dt), torch.randn(T, d, generator=g).to(dt) if pre else None
    rn, yn = _np(r), _np(y)
    total, normed = M.mote_residual_norm(block, r.cuda(), y.cuda())
    back = M.mote_residual_norm_backward(block, r.cuda(), y.cuda(), d_total.cuda(), None if d_normed is None else d_normed.cuda())
    torch.cuda.synchronize()
    t_ref, n_ref = O.residual_norm(rn, yn, **ora)
    z_mag, t_mag, n_mag, hat_y, hat, inv_y, inv = _magnitudes(rn, yn, ora)
    _close(total, t_ref, HALF[dt] * np.abs(t_ref) + 64 * U * t_mag + TINY, "total")
    if pre is None:
        assert normed is None
    else:
        _close(normed, n_ref, HALF[dt] * np.abs(n_ref) + 64 * U * n_mag + TINY, "normed")
    ref = O.residual_norm_backward(rn, yn, _np(d_total), _np(d_normed), **ora)
    mean = lambda v: v.mean(axis=1, keepdims=True)
    up = np.abs(_np(d_total))
    if pre is not None:
        u = np.abs(_np(d_normed)) * np.abs(ora["pre"][1])
        up = up + inv * (1 + inv * np.sqrt(mean(t_mag ** 2))) * (u + mean(u) + hat * mean(u * hat))
    _close(back.dr, ref["dr"], HALF[dt] * np.abs(ref["dr"]) + 256 * U * 0.75 * up + TINY, "dr")
    dz = 0.5 * up * (1.0 if ora["gate"] is None else np.abs(ora["gate"]))
    dy = dz
    if post is not None:
        v = dz * np.abs(ora["post"][1])
        dy = inv_y * (v + mean(v) + hat_y * mean(v * hat_y))
    _close(back.dy, ref["dy"], HALF[dt] * np.abs(ref["dy"]) + 256 * U * dy + TINY, "dy")
    sums = dict(gate=(0.5 * z_mag * up), post_gamma=dz * hat_y, post_beta=dz, pre_gamma=0 if pre is None else np.abs(_np(d_normed)) * hat,
                pre_beta=0 if pre is None else np.abs(_np(d_normed)))
    for n, m in sums.items():
        got = getattr(back, n)
        assert (got is None) == (ref[n] is None), n
        if got is not None:
            _close(got, ref[n], (256 + T) * U * m.sum(axis=0) + TINY, n)


def test_residual_gradient_of_one_output_only():
    g = torch.Generator().manual_seed(5)
    T, d = 37, 640
    block, ora = _block(d, "rms", "layer", True, g)
    r, y, dt, dn = (torch.randn(T, d, generator=g).cuda() for _ in range(4))
    zero = torch.zeros_like(dt)
    for a, b in (((dt, None), (dt, zero)), ((None, dn), (zero, dn)), ((None, None), (zero, zero))):
        for p, q in zip(M.mote_residual_norm_backward(block, r, y, *a), M.mote_residual_norm_backward(block, r, y, *b)):
            assert (p is None and q is None) or torch.equal(p, q)
    both = M.mote_residual_norm_backward(block, r, y, dt, dn)
    lean = M.mote_residual_norm_backward(block, r, y, dt, dn, want_params=False)
    assert torch.equal(both.dr, lean.dr) and torch.equal(both.dy, lean.dy) and all(v is None for v in lean[2:])


@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer")])
def test_residual_gradient_without_eps_of_a_ragged_batch(post, pre):
    """eps = 0: what a workgroup has behind the last row must not reach the sums (its scale would be infinite)."""
    g = torch.Generator().manual_seed(12)
    for T, d in ((1, 64), (3, 520), (5, 264), (1, 8), (2, 3000)):
        block, ora = _block(d, post, pre, True, g, eps=0.0)
        r, y, dt, dn = (torch.randn(T, d, generator=g) for _ in range(4))
        back = M.mote_residual_norm_backward(block, r.cuda(), y.cuda(), dt.cuda(), dn.cuda())
        ref = O.residual_norm_backward(_np(r), _np(y), _np(dt), _np(dn), **ora)
        for n in ("dr", "dy", "gate", "post_gamma", "pre_gamma"):
            got = _np(getattr(back, n))
            assert np.linalg.norm(got - ref[n]) <= 512 * U * np.linalg.norm(ref[n]) * d ** 0.5 + TINY, (T, d, n)


def test_residual_rows_of_zeros_constants_and_nonfinite_values():
    g = torch.Generator().manual_seed(6)
    T, d = 12, 896
    block, ora = _block(d, "layer", "rms", True, g, eps=1e-5)
    r, y = torch.randn(T, d, generator=g), torch.randn(T, d, generator=g)
    r[0], y[0] = 0.0, 0.0
    y[1] = 2.0                                  # no variance
    r[2], y[3] = 1e-20, 1e-20
    dt, dn = torch.randn(T, d, generator=g), torch.randn(T, d, generator=g)
    total, normed = M.mote_residual_norm(block, r.cuda(), y.cuda())
    t_ref, n_ref = O.residual_norm(_np(r), _np(y), **ora)
    m = _magnitudes(_np(r), _np(y), ora)
    _close(total, t_ref, U * np.abs(t_ref) + 64 * U * m[1] + TINY, "total")
    _close(normed, n_ref, U * np.abs(n_ref) + 64 * U * m[2] + TINY, "normed")
    back = M.mote_residual_norm_backward(block, r.cuda(), y.cuda(), dt.cuda(), dn.cuda())
    assert all(torch.isfinite(t).all() for t in back if t is not None)
    r2 = r.clone()
    r2[5, 7], r2[6, 0] = math.nan, math.inf      # stays in its row
    total2, normed2 = M.mote_residual_norm(block, r2.cuda(), y.cuda())
    keep = [i for i in range(T) if i not in (5, 6)]
    assert torch.equal(total2[keep], total[keep]) and torch.equal(normed2[keep], normed[keep]) and normed2[5].isnan().all()


def test_residual_writes_nothing_behind_the_last_row():
    g = torch.Generator().manual_seed(8)
    for T, d in ((1, 264), (5, 128), (3, 8), (6, 1032)):
        block, _ = _block(d, "rms", "rms", True, g)
        buf = [torch.full((T + 5, d), 7.0, device="cuda") for _ in range(2)]
        r, y = torch.randn(T, d, generator=g).cuda(), torch.randn(T, d, generator=g).cuda()
        M.mote_residual_norm(block, r, y, total=buf[0][:T], normed=buf[1][:T])
        torch.cuda.synchronize()
        assert all((b[T:] == 7.0).all() and (b[:T] != 7.0).any() for b in buf)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 8), (37, 264), (5000, 1032), (3, 8192)])
def test_residual_in_place(T, d, dt):
    """Outputs in the place of the inputs: the same bits as in memory of their own."""
    g = torch.Generator().manual_seed(T + d)
    block, _ = _block(d, "layer", "rms", True, g)
    r, y = torch.randn(T, d, generator=g).cuda().to(dt), torch.randn(T, d, generator=g).cuda().to(dt)
    want = M.mote_residual_norm(block, r, y)
    for into_r in (True, False):
        r2, y2 = r.clone(), y.clone()
        total, normed = (r2, y2) if into_r else (y2, r2)
        got = M.mote_residual_norm(block, r2, y2, total=total, normed=normed)
        torch.cuda.synchronize()
        assert got[0] is total and got[1] is normed
        assert torch.equal(total, want[0]) and torch.equal(normed, want[1]), into_r


def test_residual_norm_of_no_rows():
    g = torch.Generator().manual_seed(9)
    block, _ = _block(256, "rms", "layer", True, g)
    e = torch.zeros(0, 256, dtype=torch.bfloat16, device="cuda")
    total, normed = M.mote_residual_norm(block, e, e)
    back = M.mote_residual_norm_backward(block, e, e, e, e)
    torch.cuda.synchronize()
    assert total.shape == normed.shape == (0, 256) and all((p == 0).all() for p in back[2:] if p is not None)


def test_residual_feeds_the_block():
    """total and normed of the call in front of a block are what mote_block_forward adds and normalises: its LN(x^a) differs
    by the rounding of x^a only."""
    cfg = W.MoteConfig("feeds", 256, 512, 4, 2, 50, seed=4)
    gp = GpuProblem(cfg)
    g = torch.Generator().manual_seed(10)
    gamma = (1 + 0.1 * torch.randn(256, generator=g)).to(torch.bfloat16).cuda()
    block = M.MoteResidual(256, pre=M.MoteNorm(gamma))
    y = torch.randn(50, 256, generator=g).to(torch.bfloat16).cuda()
    total, normed = M.mote_residual_norm(block, gp.x, y)
    taps = M.alloc_taps(gp.layer, 50, ("xn",))
    M.mote_block_forward(gp.layer, total, gamma, taps=taps)
    # one rounding of each input and one of the output, each 2^-8 of the value, and of the row's scale
    assert ((taps["xn"].float() - normed.float()).abs() <= 3 * 2.0 ** -8 * normed.float().abs() + TINY).all()


# ----------------------------------------------------------------------------------------------------------- clipping
def _check_clip(grads, max_norm, in_place, outs=None):
    dev = [t.cuda() for t in grads]
    keep = [t.clone() for t in dev]
    outs = None if in_place else ([torch.full_like(t, 9.0) for t in dev] if outs is None else outs)
    clip = M.GradClip(dev, outs)
    norm = M.mote_clip_grad_norm(clip, max_norm)
    torch.cuda.synchronize()
    n_ref, ref = O.clip_grad_norm([_np(t) for t in grads], float(np.float32(max_norm)))
    if n_ref < 3.4028235e38:
        assert abs(norm.item() - n_ref) <= 2 * U * n_ref + TINY
    else:                                              # not finite, or beyond the largest fp32 value
        assert not math.isfinite(norm.item())
    res = dev if in_place else outs
    for got, want, src in zip(res, ref, grads):
        if not np.isfinite(n_ref) or n_ref <= max_norm * (1 - 1e-12):
            assert torch.equal(got.cpu().view(torch.int16 if src.dtype == torch.bfloat16 else torch.int32),
                               src.view(torch.int16 if src.dtype == torch.bfloat16 else torch.int32))
        else:                                          # the product rounded to fp32, then to the type
            _close(got, want, (HALF[src.dtype] + 4 * U) * np.abs(want) + 1e-40, "scaled")
    if not in_place:
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(dev, keep))   # bits: NaN is not equal to itself
    return norm


def _grads(sizes, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * scale).to(torch.bfloat16 if i % 3 == 1 else torch.float32) for i, n in enumerate(sizes)]


@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [7, 8, 9], [16383, 16384, 16385], [1, 2, 3, 5, 40000, 100003], [64] * 119, [33] * 120, [65] * 121, [17] * 400,
                                   [5000000], [0]])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_sizes(sizes, in_place):
    grads = _grads(sizes, len(sizes) + sum(sizes))
    total = max(sum(sizes), 1)
    for limit in (0.3 * math.sqrt(total), 10 * math.sqrt(total), math.inf):
        _check_clip(grads, limit, in_place)


def test_clip_alignment_of_views():
    """Gradients and outputs that start at any element of a flat buffer, aligned to their type only, next to each other."""
    g = torch.Generator().manual_seed(2)
    for dt in (torch.float32, torch.bfloat16):
        flat = torch.randn(100000, generator=g).to(dt).cuda()
        keep, out = flat.clone(), torch.full((100010,), 9.0, dtype=dt, device="cuda")
        cuts = [0, 1, 2, 5, 12, 1000, 1003, 20011, 20011, 57777, 99999]
        views = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
        outs = [out[a + 3:b + 3] for a, b in zip(cuts, cuts[1:])]
        norm = M.mote_clip_grad_norm(M.GradClip(views, outs), 1.0)
        n_ref, (ref,) = O.clip_grad_norm([_np(keep[:99999])], 1.0)
        assert abs(norm.item() - n_ref) <= 2 * U * n_ref
        _close(out[3:100002], ref, (HALF[dt] + 4 * U) * np.abs(ref) + 1e-40, "scaled")
        assert (out[:3] == 9).all() and (out[100002:] == 9).all() and torch.equal(flat, keep)
        M.mote_clip_grad_norm(M.GradClip(views), 1.0)               # and in place: the same, nothing behind the last
        assert torch.equal(flat[:99999], out[3:100002]) and flat[99999] == keep[99999]


def test_clip_values():
    _check_clip(_grads([1000, 1000], 3, 1e30), 1.0, False)          # squares beyond fp32
    _check_clip(_grads([1000, 1000], 3, 1e-30), 1e-29, True)        # squares below fp32
    _check_clip([torch.zeros(100)], 1.0, True)
    _check_clip([torch.full((4,), 3e38)], 1.0, False)               # a norm beyond fp32: reported as inf, still scaled
    for v in (math.inf, -math.inf, math.nan):
        t = torch.randn(5000)
        t[4321] = v
        _check_clip([torch.randn(10), t], 1.0, True)
        _check_clip([torch.randn(10), t], 1.0, False)


def test_clip_is_the_same_every_time():
    clip = M.GradClip([t.cuda() for t in _grads([100003, 77, 50021, 3], 8)], [t.cuda() for t in _grads([100003, 77, 50021, 3], 9)])
    first = M.mote_clip_grad_norm(clip, 1.0)
    outs = [o.clone() for o in clip.outs]
    for _ in range(5):
        assert torch.equal(M.mote_clip_grad_norm(clip, 1.0), first) and all(torch.equal(a, b) for a, b in zip(outs, clip.outs))


# -------------------------------------------------------------------------------- streams, graphs, refusals, together
class _Step:
    """One training step's operators around a layer, on buffers of its own: route, layer on the routing, residual and norms,
    their gradients, the router's gradient, clipping of all parameter gradients."""

    def __init__(self, T, seed):
        self.cfg = W.MoteConfig("step", 256, 512, 8, 2, T, seed=seed)
        self.gp = GpuProblem(self.cfg)
        g = torch.Generator().manual_seed(seed)
        self.x = self.gp.x.clone()
        self.block, _ = _block(256, "rms", "rms", True, g)
        self.routing = M.MoteRouting(2, score="sigmoid", n_groups=4, top_groups=2, group_top=2, renormalise=True)
        self.bias = (torch.randn(8, generator=g) * 0.02).cuda()
        self.mask = torch.ones(T, dtype=torch.uint8, device="cuda")
        self.mask[T - T // 4:] = 0
        self.d_w = torch.randn(T, 2, generator=g).cuda()
        self.up = torch.randn(T, 256, generator=g).to(torch.bfloat16).cuda()
        self.layer_ws = torch.empty(self.gp.layer.workspace_bytes(T), dtype=torch.uint8, device="cuda")

    def __call__(self):
        r = M.mote_route(self.x, self.gp.w_router, self.routing, select_bias=self.bias, token_mask=self.mask, want_logits=True, want_stats=True)
        y = M.mote_layer_forward_routed(self.gp.layer, self.x, r.topk_idx, r.topk_w, workspace=self.layer_ws)
        total, normed = M.mote_residual_norm(self.block, self.x, y)
        back = M.mote_residual_norm_backward(self.block, self.x, y, self.up, self.up)
        q = r.counts.float() * (0.01 * 8 / self.x.shape[0])
        dx, dw = M.mote_route_backward(self.x, self.gp.w_router, self.routing, r.logits, r.topk_idx, self.d_w, q, self.mask)
        grads = [dw] + [p for p in back[2:] if p is not None]
        outs = [torch.empty_like(t) for t in grads]
        norm = M.mote_clip_grad_norm(M.GradClip(grads, outs), 1.0)
        return [r.topk_idx, r.topk_w, r.logits, r.counts, r.score_sum, y, total, normed, back.dr, back.dy, dx, norm, *grads, *outs]


def test_the_operators_together_against_the_oracle():
    s = _Step(200, 21)
    (idx, wt, logits, counts, ssum, y, total, normed, dr, dy, dx, norm, dw, d_gate, d_post, d_pre, *outs) = s()
    torch.cuda.synchronize()
    x, w = _np(s.x), _np(s.gp.w_router)
    ref = O.route(x, w, 2, "sigmoid", s.bias.cpu().numpy(), s.mask.cpu().numpy(), 4, 2, 2, True)
    assert np.array_equal(idx.cpu().numpy(), ref["idx"]) and np.array_equal(counts.cpu().numpy(), ref["counts"])
    assert np.allclose(wt.cpu().numpy(), ref["w"], rtol=1e-5) and np.allclose(ssum.cpu().numpy(), ref["score_sum"], rtol=1e-5)
    want = O.layer_forward(W.bf16_bits(s.x.cpu()), W.bf16_bits(s.gp.w_router.cpu()), None, 2, [W.bf16_bits(t.cpu()) for t in s.gp.shared],
                           lambda e: tuple(v for m in range(3) for v in O.ternarize(W.make_latent(s.cfg, e, m).numpy())), tokens=np.arange(150, 200))
    assert np.abs(_np(y[150:]) - want["y_s"]).max() <= 2e-2                 # padding tokens: the shared expert alone
    blk = s.block
    ora = dict(post=("rms", _np(blk.post.gamma), None, 1e-6), gate=_np(blk.gate), pre=("rms", _np(blk.pre.gamma), None, 1e-6), residual_scale=0.75,
               branch_scale=0.5)
    t_ref, n_ref = O.residual_norm(x, _np(y), **ora)
    assert np.allclose(_np(total), t_ref, rtol=2.0 ** -8, atol=1e-5) and np.allclose(_np(normed), n_ref, rtol=2.0 ** -8, atol=1e-5)
    b = O.residual_norm_backward(x, _np(y), _np(s.up), _np(s.up), **ora)
    for got, name in ((dr, "dr"), (dy, "dy"), (d_gate, "gate"), (d_post, "post_gamma"), (d_pre, "pre_gamma")):
        assert np.linalg.norm(_np(got) - b[name]) <= 2.0 ** -8 * np.linalg.norm(b[name]), name
    q = ref["counts"] * (0.01 * 8 / 200)
    _, dx_ref, dw_ref, _ = O.route_backward(x, w, _np(logits), ref["idx"], _np(s.d_w), q, s.mask.cpu().numpy(), "sigmoid", True, 1.0)
    assert np.linalg.norm(_np(dx) - dx_ref) <= 1e-5 * np.linalg.norm(dx_ref) and np.linalg.norm(_np(dw) - dw_ref) <= 1e-5 * np.linalg.norm(dw_ref)
    n_ref, c_ref = O.clip_grad_norm([_np(t) for t in (dw, d_gate, d_post, d_pre)], 1.0)
    assert abs(norm.item() - n_ref) <= 2 * U * n_ref
    for got, c in zip(outs, c_ref):
        assert np.allclose(_np(got), c, rtol=4 * U, atol=1e-40)


@pytest.mark.parametrize("T", [1, 37, 600])
def test_captured_step_replays(T):
    s = _Step(T, 31)
    s()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s()
    g = torch.Generator().manual_seed(T)
    for i in range(4):                       # other inputs and eager work between the replays
        s.x.copy_(torch.randn(s.x.shape, generator=g).to(torch.bfloat16))
        s.bias.copy_(torch.randn(8, generator=g) * 0.05)
        want = [t.clone() for t in s()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    steps = [_Step(300, 41), _Step(280, 42)]
    want = [[t.clone() for t in s()] for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    M.mote_tuning_set("no_fork", 1)            # the layer's helper stream is shared by design
    try:
        for _ in range(3):
            got = []
            for s, st in zip(steps, streams):
                st.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(st):
                    got.append(s())
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert all(torch.equal(p, q) for p, q in zip(a, b))
    finally:
        M.mote_tuning_set("no_fork", 0)


def test_binding_refuses_shapes_types_and_strides():
    x, w = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda"), torch.zeros(256, 8, dtype=torch.bfloat16, device="cuda")
    r = M.MoteRouting(2)
    ok = M.mote_route(x, w, r, want_logits=True)
    f32 = lambda *s: torch.zeros(*s, device="cuda")
    block = M.MoteResidual(256, pre=M.MoteNorm(x[0].contiguous()))
    calls = [lambda: M.mote_route(x.float(), w, r), lambda: M.mote_route(x[:, ::2], w[:128], r), lambda: M.mote_route(x, w[:128].contiguous(), r),
             lambda: M.mote_route(x, w, r, select_bias=f32(7)), lambda: M.mote_route(x, w, r, token_mask=f32(4)),
             lambda: M.mote_route(x, w, r, token_mask=torch.zeros(5, dtype=torch.uint8, device="cuda")), lambda: M.mote_route(x, w, M.MoteRouting(9)),
             lambda: M.mote_route(x, w, M.MoteRouting(2, n_groups=3)), lambda: M.mote_route(x.cpu(), w, r),
             lambda: M.mote_route(x, w, r, want_stats=True, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")),
             lambda: M.mote_route_backward(x, w, r, ok.logits, ok.topk_idx[:3].contiguous(), ok.topk_w),
             lambda: M.mote_route_backward(x, w, r, ok.logits[:, :4].contiguous(), ok.topk_idx, ok.topk_w),
             lambda: M.mote_route_backward(x, w, r, ok.logits, ok.topk_idx.long(), ok.topk_w),
             lambda: M.mote_route_backward(x, w, r, ok.logits, ok.topk_idx, ok.topk_w, d_score_sum=f32(4)),
             lambda: M.mote_residual_norm(block, x, x.float()), lambda: M.mote_residual_norm(block, x, x[:3]),
             lambda: M.mote_residual_norm(block, x[:, :128].contiguous(), x[:, :128].contiguous()),
             lambda: M.mote_residual_norm(M.MoteResidual(256), x, x, normed=torch.empty_like(x)),
             lambda: M.mote_residual_norm_backward(M.MoteResidual(256), x, x, x, x), lambda: M.MoteResidual(256, gate=f32(256)),
             lambda: M.MoteNorm(f32(256)), lambda: M.GradClip([f32(4, 4)[:, :2]]), lambda: M.GradClip([f32(4)], [f32(5)]),
             lambda: M.GradClip([x, f32(3).half()]), lambda: M.mote_clip_grad_norm(M.GradClip([x, x]), 1.0),
             lambda: M.mote_clip_grad_norm(M.GradClip([x]), -1.0)]
    for i, f in enumerate(calls):
        with pytest.raises(M.MoteError):
            f()
            print("call", i, "went through")
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------- offsets beyond 32 bits
def test_routing_of_more_than_2_31_elements():
    """The last tokens of a batch whose rows pass 2^31 elements: the same bits as in a batch of their own that starts at a
    multiple of 32 tokens; one token with a gradient gives dw in both (zeros change no sum)."""
    T, d, E, tail = 32896, 65536, 8, 96
    g = torch.Generator(device="cuda").manual_seed(40)
    x = torch.randn(T, d, generator=g, device="cuda", dtype=torch.bfloat16)
    w = (torch.randn(d, E, generator=g, device="cuda") * d ** -0.5).bfloat16()
    last = x[-tail:].clone()
    assert x[:-tail].numel() > 2 ** 31
    cfg = M.MoteRouting(2, renormalise=True)
    a, b = M.mote_route(x, w, cfg, want_logits=True, want_stats=True), M.mote_route(last, w, cfg, want_logits=True)
    assert torch.equal(a.topk_idx[-tail:], b.topk_idx) and torch.equal(a.topk_w[-tail:], b.topk_w) and torch.equal(a.logits[-tail:], b.logits)
    assert int(a.counts.sum()) == 2 * T
    d_w = torch.zeros(T, 2, device="cuda")
    d_w[-1] = torch.tensor([0.75, -0.5], device="cuda")
    dx, dw = M.mote_route_backward(x, w, cfg, a.logits, a.topk_idx, d_w)
    dx_b, dw_b = M.mote_route_backward(last, w, cfg, b.logits, b.topk_idx, d_w[-tail:].clone())
    torch.cuda.synchronize()
    assert torch.equal(dx[-tail:], dx_b) and (dx_b[-1] != 0).any() and not (dx[:8] != 0).any()
    assert torch.equal(dw, dw_b) and (dw_b != 0).any()


def test_residual_of_more_than_2_31_elements():
    T, d, tail = 262400, 8192, 200
    g = torch.Generator().manual_seed(41)
    block, _ = _block(d, "rms", "layer", True, g)
    gpu = torch.Generator(device="cuda").manual_seed(42)
    r, y = (torch.randn(T, d, generator=gpu, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    assert r[:-tail].numel() > 2 ** 31
    total, normed = M.mote_residual_norm(block, r, y)
    want = M.mote_residual_norm(block, r[-tail:].clone(), y[-tail:].clone())
    assert torch.equal(total[-tail:], want[0]) and torch.equal(normed[-tail:], want[1])
    back = M.mote_residual_norm_backward(block, r, y, total, normed, want_params=False)
    want = M.mote_residual_norm_backward(block, r[-tail:].clone(), y[-tail:].clone(), want[0], want[1], want_params=False)
    torch.cuda.synchronize()
    assert torch.equal(back.dr[-tail:], want.dr) and torch.equal(back.dy[-tail:], want.dy)


def test_clip_of_more_than_2_31_elements():
    """Only the ends of a tensor and another tensor are not zero: 3-4-12 gives 13, and every coefficient is 1 / 2."""
    n = 2 ** 31 + 8195
    g, other = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.full((1,), 12.0, device="cuda")
    g[0], g[-1] = 3.0, 4.0
    norm = M.mote_clip_grad_norm(M.GradClip([g, other]), 6.5)
    torch.cuda.synchronize()
    assert norm.item() == 13.0 and g[0].item() == 1.5 and g[-1].item() == 2.0 and other.item() == 6.0
    assert int((g != 0).sum()) == 2
