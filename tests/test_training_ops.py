"""CPU checks of the training-step operators (scored routing, residual with norms, gradient clipping): the oracle against
differences and hand-worked cases, and the argument checks of the library, which refuse a call before anything touches a
device."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2506_14435_amd as M
from oracle import mote_oracle as O

B = M.binding
P = 256                                    # a pointer that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(M.LIB_PATH):
        from paper_2506_14435_amd import build
        build.build()
    return M.load_library()


# ----------------------------------------------------------------------------------------------- the oracle itself
def test_route_worked_by_hand():
    x = np.eye(4)[:2]                       # logits are rows of w
    w = np.array([[1.0, 3.0, 2.0, 2.0], [0.0, 0.0, 0.0, 0.0], [0, 0, 0, 0], [0, 0, 0, 0]])
    r = O.route(x, w, 3)
    assert r["idx"].tolist() == [[1, 2, 3], [0, 1, 2]]              # descending, ties to the lower index
    e = np.exp([1.0, 3.0, 2.0, 2.0])
    assert np.allclose(r["w"][0], (e / e.sum())[[1, 2, 3]], rtol=1e-15)
    assert r["counts"].tolist() == [1, 2, 2, 1]
    # the bias selects, the weights do not see it; -inf switches off
    r = O.route(x, w, 2, "sigmoid", select_bias=np.array([1.0, 0, 0, -np.inf]), renormalise=True, scale=2.5)
    s = 1 / (1 + np.exp(-np.array([1.0, 3.0, 2.0])))
    assert r["idx"].tolist() == [[0, 1], [0, 1]]
    assert np.allclose(r["w"][0], 2.5 * s[:2] / s[:2].sum(), rtol=1e-14) and np.allclose(r["w"][1], 1.25, rtol=1e-14)
    # two groups of two: sums of both keys 4 against 4 -> the lower group; the best single key wins otherwise
    assert O.route(x, w, 2, n_groups=2, top_groups=1, group_top=1)["idx"][0].tolist() == [1, 0]
    off = O.route(x, w, 3, "softmax", select_bias=np.array([0, -np.inf, -np.inf, -np.inf]), renormalise=True)
    assert off["idx"][0].tolist() == [0, -1, -1] and off["w"][0].tolist() == [1.0, 0.0, 0.0]
    none = O.route(x, w, 2, token_mask=np.array([1, 0]))
    assert none["idx"][1].tolist() == [-1, -1] and none["counts"].sum() == 2


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_gradient_is_that_of_differences(score, renormalise):
    rng = np.random.default_rng(5)
    T, d, E, k, scale = 4, 6, 5, 3, 1.7
    x, w = rng.standard_normal((T, d)), rng.standard_normal((d, E))
    idx = O.route(x, w, k, score)["idx"]
    idx[1, 2] = -1                          # an empty slot
    idx[2] = [3, 3, 1]                      # one expert twice
    idx[3] = -1
    d_w, q, mask = rng.standard_normal((T, k)), rng.standard_normal(E), np.array([1, 1, 1, 0])
    g, dx, dw, mag = O.route_backward(x, w, x @ w, idx, d_w, q, mask, score, renormalise, scale)
    assert (np.abs(g) <= mag * (1 + 1e-12)).all()
    f = lambda a, b: O.route_loss(a @ b, idx, d_w, q, mask, score, renormalise, scale)
    h = 1e-6                                # central differences: error h^2 and 1e-16 / h, both below 1e-9
    for t in range(T):
        for c in range(d):
            step = np.zeros_like(x)
            step[t, c] = h
            assert abs((f(x + step, w) - f(x - step, w)) / (2 * h) - dx[t, c]) < 1e-8
    for c in range(d):
        for e in range(E):
            step = np.zeros_like(w)
            step[c, e] = h
            assert abs((f(x, w + step) - f(x, w - step)) / (2 * h) - dw[c, e]) < 1e-8


@pytest.mark.parametrize("post,pre,gated", [("rms", "layer", True), ("layer", "rms", True), (None, "rms", False), ("layer", None, True),
                                            (None, None, True)])
def test_residual_gradient_is_that_of_differences(post, pre, gated):
    rng = np.random.default_rng(7)
    T, d = 3, 8
    par = {n: rng.standard_normal(d) for n in ("gate", "post_gamma", "post_beta", "pre_gamma", "pre_beta")}
    data = dict(r=rng.standard_normal((T, d)), y=rng.standard_normal((T, d)), **par)
    d_total, d_normed = rng.standard_normal((T, d)), rng.standard_normal((T, d)) if pre else None

    def block(v):
        return dict(post=post and (post, v["post_gamma"], v["post_beta"], 1e-3), gate=v["gate"] if gated else None,
                    pre=pre and (pre, v["pre_gamma"], v["pre_beta"], 1e-3), residual_scale=0.75, branch_scale=0.5)

    def f(v):
        total, normed = O.residual_norm(v["r"], v["y"], **block(v))
        return (total * d_total).sum() + ((normed * d_normed).sum() if pre else 0.0)

    got = O.residual_norm_backward(data["r"], data["y"], d_total, d_normed, **block(data))
    for name, grad in (("r", got["dr"]), ("y", got["dy"]), *[(n, got[n]) for n in par]):
        if grad is None:
            continue
        for i in np.ndindex(grad.shape):
            up, down = dict(data), dict(data)
            up[name], down[name] = data[name].copy(), data[name].copy()
            up[name][i] += 1e-6
            down[name][i] -= 1e-6
            assert abs((f(up) - f(down)) / 2e-6 - grad[i]) < 1e-8, (name, i)


def test_clip_worked_by_hand():
    norm, out = O.clip_grad_norm([np.array([3.0]), np.array([0.0, 4.0])], 1.0)
    assert norm == 5.0 and out[0][0] == 0.6000000000000001 and out[1][1] == 0.8
    assert O.clip_grad_norm([np.array([3.0, 4.0])], 5.0)[1][0].tolist() == [3.0, 4.0]
    norm, out = O.clip_grad_norm([np.array([np.inf, 1.0])], 1.0)
    assert norm == np.inf and out[0][1] == 1.0


# -------------------------------------------------------------------------------------------------------- refusals
def _routing(**kw):
    v = dict(score=0, top_k=2, n_groups=1, top_groups=1, group_top=1, renormalise=0, scale=1.0)
    v.update(kw)
    return ctypes.byref(B.MoteRoutingStruct(*v.values()))


def test_route_refuses_on_the_host(lib):
    def call(T=4, d=256, E=8, x=P, w=P, idx=P, wt=P, counts=None, ws=P, ws_bytes=1 << 20, **cfg):
        return lib.mote_route(_routing(**cfg), x, w, None, None, T, d, E, idx, wt, None, counts, None, ws, ws_bytes, None)

    assert lib.mote_route(None, P, P, None, None, 4, 256, 8, P, P, None, None, None, P, 1 << 20, None) == 1
    for bad in (dict(T=-1), dict(score=2), dict(scale=math.inf), dict(scale=math.nan), dict(n_groups=0), dict(n_groups=3), dict(n_groups=16),
                dict(n_groups=4, top_groups=0), dict(n_groups=4, top_groups=5), dict(n_groups=4, top_groups=2, group_top=3), dict(x=None),
                dict(w=None), dict(idx=None), dict(wt=None), dict(counts=P, ws=None), dict(counts=P, ws=P + 16)):
        assert call(**bad) == 1, bad
    for bad in (dict(d=200), dict(d=0), dict(E=0), dict(E=65), dict(top_k=0), dict(top_k=9, E=16), dict(top_k=5, E=4), dict(T=1 << 23),
                dict(n_groups=8, top_groups=2, group_top=2), dict(n_groups=4, top_groups=1, top_k=3)):
        assert call(**bad) == 2, bad
    assert call(counts=P, ws_bytes=64) == 3
    assert call(T=0, x=None, w=None, idx=None, wt=None) == 0          # nothing to do
    assert lib.mote_route_workspace_bytes(-1, 256, 8) == 0 and lib.mote_route_workspace_bytes(4, 256, 65) == 0
    assert lib.mote_route_workspace_bytes(4, 100, 8) == 0 and lib.mote_route_workspace_bytes(0, 256, 8) > 0
    assert call(T=65, ws=None) == 1 and call(T=65, ws_bytes=1024) == 3     # the laid out weights


def test_route_backward_refuses_on_the_host(lib):
    def call(T=4, d=256, E=8, x=P, w=P, logits=P, idx=P, d_w=P, dx=P, dw=P, ws=P, ws_bytes=1 << 24, **cfg):
        return lib.mote_route_backward(_routing(**cfg), x, w, logits, idx, d_w, None, None, T, d, E, dx, dw, ws, ws_bytes, None)

    for bad in (dict(T=-1), dict(score=7), dict(x=None), dict(w=None), dict(logits=None), dict(idx=None), dict(d_w=None), dict(ws=None),
                dict(ws=P + 8)):
        assert call(**bad) == 1, bad
    for bad in (dict(d=64), dict(E=65), dict(top_k=9), dict(T=1 << 23)):
        assert call(**bad) == 2, bad
    assert call(ws_bytes=16) == 3
    assert call(dx=None, dw=None, ws=None) == 0                        # nothing asked for
    assert lib.mote_route_backward_workspace_bytes(4, 100, 8) == 0


def _norm(kind=1, gamma=P, beta=None, eps=1e-6):
    return ctypes.pointer(B.MoteNormStruct(kind, gamma, beta, eps))


def test_residual_refuses_on_the_host(lib):
    def block(post=None, gate=None, a=1.0, b=1.0, pre=None):
        return ctypes.byref(B.MoteResidualStruct(post, gate, a, b, pre))

    def call(blk, r=P, y=P, dtype=1, T=4, d=64, total=P, normed=P):
        return lib.mote_residual_norm(blk, r, y, dtype, T, d, total, normed, None)

    ok = block(pre=_norm())
    assert call(None) == 1
    for bad in (dict(dtype=2), dict(T=-1), dict(r=None), dict(y=None), dict(total=None), dict(normed=None)):
        assert call(ok, **bad) == 1, bad
    for bad in (dict(d=60), dict(d=0), dict(d=8200)):
        assert call(ok, **bad) == 2, bad
    for bad in (dict(post=_norm(kind=3)), dict(post=_norm(gamma=None)), dict(pre=_norm(kind=2)), dict(pre=_norm(eps=-1.0)),
                dict(pre=_norm(eps=math.nan)), dict(a=math.nan), dict(b=math.inf)):
        assert call(block(**bad)) == 1, bad
    assert call(ok, T=0, r=None, y=None, total=None) == 0

    def back(blk, r=P, y=P, dt=P, dn=P, T=4, d=64, dr=P, dy=P, ws=P, n=1 << 20):
        return lib.mote_residual_norm_backward(blk, r, y, dt, dn, 1, T, d, dr, dy, None, ws, n, None)

    for bad in (dict(r=None), dict(y=None), dict(dr=None), dict(dy=None), dict(ws=None), dict(ws=P + 4)):
        assert back(ok, **bad) == 1, bad
    assert back(block()) == 1                                           # a gradient of an output that is not there
    assert back(ok, n=0) == 3 and back(ok, d=60) == 2
    assert lib.mote_residual_norm_workspace_bytes(ok, 4, 60) == 0


def test_clip_refuses_on_the_host(lib):
    def call(*tensors, max_norm=1.0, norm=P, ws=P, ws_bytes=1 << 20, n=None):
        arr = (B.MoteGradStruct * max(len(tensors), 1))(*[B.MoteGradStruct(*t) for t in tensors])
        return lib.mote_clip_grad_norm(arr, len(tensors) if n is None else n, max_norm, norm, ws, ws_bytes, None)

    good = (0x1000, None, 16, 0)
    for bad in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(norm=None), dict(ws=None), dict(ws=P + 1), dict(n=-1)):
        assert call(good, **bad) == 1, bad
    assert call(good, n=4097) == 2 and call(good, ws_bytes=8) == 3
    assert lib.mote_clip_grad_norm(None, 1, 1.0, P, P, 1 << 20, None) == 1
    for bad in ((0x1000, None, -1, 0), (0x1000, None, 4, 5), (None, None, 4, 0), (0x1002, None, 4, 0), (0x1001, None, 4, 1), (0x1000, 0x2002, 4, 0)):
        assert call(bad) == 1, bad
    assert call((0x1000, None, 1 << 40, 0)) == 2
    # overlaps: the same tensor twice, an output on another's gradient, partly overlapping outputs, an output on its own gradient shifted
    for bad in ([good, good], [good, (0x2000, 0x1020, 4, 0)], [(0x1000, 0x8000, 8, 0), (0x2000, 0x8010, 8, 1)], [(0x1000, 0x1004, 8, 0)],
                [(0x1000, None, 100, 0), (0x5000, None, 1, 0), (0x1010, 0x9000, 1, 1)]):
        assert call(*bad) == 1, bad
    assert lib.mote_clip_grad_norm_workspace_bytes(-1) == 0 and lib.mote_clip_grad_norm_workspace_bytes(4097) == 0


def test_workspace_sizes_at_the_ends_of_the_range(lib):
    """Token counts that the calls refuse have no workspace; sizes do not fall as the count grows to the largest."""
    for f in (lib.mote_route_workspace_bytes, lib.mote_route_backward_workspace_bytes):
        for T in (1 << 24, (1 << 31) - 600, (1 << 31) - 1):
            assert f(T, 256, 8) == 0, T
        sizes = [f(T, 256, 8) for T in (1, 64, 65, 5000, 1 << 20, (1 << 24) - 1)]
        assert sizes == sorted(sizes) and sizes[-1] > 0
    block = ctypes.byref(B.MoteResidualStruct(None, None, 1.0, 1.0, _norm()))
    sizes = [lib.mote_residual_norm_workspace_bytes(block, T, 8) for T in (1, 1000, 1 << 20, (1 << 31) - 1)]
    assert sizes == sorted(sizes)


def test_overlap_check_allows_what_does_not_overlap(lib):
    """Gradients that are only read may share memory, neighbours may touch.  The workspace is checked last: a list that passes
    ends there, before any launch."""
    for tensors in ([(0x1000, 0x8000, 8, 0), (0x1000, 0x9000, 8, 0)], [(0x1000, None, 4, 0), (0x1010, None, 4, 0)],
                    [(0x1010, 0x1000, 4, 0)], [(0x1000, None, 0, 0), (0x1000, None, 4, 0)]):
        arr = (B.MoteGradStruct * len(tensors))(*[B.MoteGradStruct(*t) for t in tensors])
        assert lib.mote_clip_grad_norm(arr, len(tensors), 1.0, P, P, 8, None) == 3, tensors


def test_binding_refuses_what_is_not_a_device_tensor():
    x, w = torch.zeros(4, 256, dtype=torch.bfloat16), torch.zeros(256, 8, dtype=torch.bfloat16)
    for f in (lambda: M.mote_route(x, w, M.MoteRouting(2)), lambda: M.MoteNorm(x[0]), lambda: M.GradClip([x]), lambda: M.GradClip([]),
              lambda: M.MoteRouting(2, score="cosine"), lambda: M.mote_residual_norm(M.MoteResidual(256), x, x),
              lambda: M.mote_residual_norm(M.MoteResidual(256), x.half(), x.half())):
        with pytest.raises(M.MoteError):
            f()
