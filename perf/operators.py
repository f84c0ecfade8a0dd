"""Cases of the training-step operators around the MoTE layer: scored routing and its gradient, the residual sum with the
norms on both sides of it and its gradient, and the clipping of gradients by their global norm.

`own` False computes them in plain torch operations (fp32, fp64 where a rounding could turn a choice), `own` True through
the library's entry points.  `exact` is the definition in fp64, written apart from the plain form."""
import math
import random

import numpy as np
import torch

own = False


# ----------------------------------------------------------------------------------------------------------- cases
def _route(name, T, d, E, k, score, bias=False, groups=1, top_groups=1, group_top=1, renorm=False, scale=1.0, off=0, mask=False,
           train=False, outliers=0):
    return dict(name=name, op="route", T=T, d=d, E=E, k=k, score=score, bias=bias, groups=groups, top_groups=top_groups,
                group_top=group_top, renorm=renorm, scale=scale, off=off, mask=mask, train=train, outliers=outliers)


def _route_bwd(name, T, d, E, k, score, renorm=False, scale=1.0, mask=False, balance=True):
    return dict(name=name, op="route_backward", T=T, d=d, E=E, k=k, score=score, renorm=renorm, scale=scale, mask=mask, balance=balance)


def _norm(name, op, T, d, post, pre, gate, dtype="bf16", residual_scale=1.0, branch_scale=1.0):
    return dict(name=name, op=op, T=T, d=d, post=post, pre=pre, gate=gate, dtype=dtype, residual_scale=residual_scale,
                branch_scale=branch_scale)


def _clip(name, kind, sizes_seed, n, lo, hi, d=0, d_ff=0, E=0, clips=True, in_place=False):
    return dict(name=name, op="clip", kind=kind, sizes_seed=sizes_seed, n=n, lo=lo, hi=hi, d=d, d_ff=d_ff, E=E, clips=clips, in_place=in_place)


def listed():
    return [
        # one token of a decode step of the 3B-width layer with 16 experts: launch and load latency
        _route("route_one_token", 1, 2048, 16, 2, "sigmoid", bias=True, renorm=True),
        # a decode batch of the 7B width, 64 experts in 8 groups, two of them switched off by their bias
        _route("route_decode_groups", 64, 3584, 64, 8, "sigmoid", bias=True, groups=8, top_groups=4, group_top=2, renorm=True, scale=2.5, off=2),
        # a training batch of the 3B width, 64 experts: logits kept for the backward pass, counts and score sums for the balance
        _route("route_train_3b", 8192, 2048, 64, 6, "softmax", renorm=True, train=True),
        # a ragged batch of the 7B width with padding tokens and outlier channels in the hidden state
        _route("route_padded_7b", 16301, 3584, 60, 4, "sigmoid", bias=True, groups=6, top_groups=3, group_top=1, renorm=True, mask=True,
               train=True, outliers=4),
        # gradient of the 0.5B width's router, eight experts, the paper's weights (not renormalised) and the balance loss
        _route_bwd("route_backward_05b", 2048, 896, 8, 2, "softmax"),
        # gradient of a wide router over a large batch with padding
        _route_bwd("route_backward_3b", 16000, 2048, 64, 8, "sigmoid", renorm=True, scale=2.5, mask=True),
        # one token: the norms around a decode step's branch
        _norm("norm_one_token", "norm", 1, 2048, "rms", "rms", True),
        # a prefill batch of the 7B width: norm behind the branch, gate, residual, norm in front of the next
        _norm("norm_prefill_7b", "norm", 16384, 3584, "rms", "rms", True, branch_scale=0.5),
        # a ragged training batch of the 3B width, layer normalisation in front of the next branch
        _norm("norm_backward_3b", "norm_backward", 8191, 2048, "rms", "layer", True, residual_scale=0.75),
        # fp32 activations of a narrow block, a norm in front only
        _norm("norm_backward_fp32", "norm_backward", 1000, 896, "none", "rms", False, dtype="f32"),
        # gradients of a small layer: a few tensors that fit the caches
        _clip("clip_small_layer", "layer", 0, 0, 0, 0, d=256, d_ff=512, E=4),
        # gradients of the 0.5B-width layer with eight experts (fp32 latent gradients, bf16 shared expert)
        _clip("clip_05b_layer", "layer", 0, 0, 0, 0, d=896, d_ff=4864, E=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route", "route_backward", "norm", "norm_backward", "clip"])
    T = _log_int(rng, 1, 16384)
    if op in ("route", "route_backward"):
        d = 128 * rng.randint(2, 28)
        E = _log_int(rng, 4, 64)
        score, renorm, scale = rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5, rng.choice([1.0, 2.5, 0.7])
        if op == "route_backward":
            return _route_bwd(None, T, d, E, rng.randint(1, min(E, 8)), score, renorm, scale, rng.random() < 0.3, rng.random() < 0.5)
        divisors = [g for g in range(1, E + 1) if E % g == 0 and E // g >= 2]
        groups = rng.choice(divisors) if rng.random() < 0.5 else 1
        top_groups = rng.randint(1, groups)
        bias = rng.random() < 0.6
        return _route(None, T, d, E, rng.randint(1, min(8, top_groups * (E // groups))), score, bias, groups, top_groups, rng.randint(1, 2),
                      renorm, scale, rng.randint(0, 2) if bias else 0, rng.random() < 0.3, rng.random() < 0.5, rng.choice([0, 4]))
    if op in ("norm", "norm_backward"):
        return _norm(None, op, T, 8 * rng.randint(16, 448), rng.choice(["none", "rms", "layer"]),
                     rng.choice(["none", "rms", "layer"]) if op == "norm" else rng.choice(["rms", "layer"]), rng.random() < 0.6,
                     rng.choice(["bf16", "bf16", "f32"]), rng.choice([1.0, 0.75]), rng.choice([1.0, 0.5]))
    if rng.random() < 0.5:
        clips = rng.random() < 0.7
        return _clip(None, "ragged", rng.randint(0, 1 << 20), _log_int(rng, 1, 400), 1, _log_int(rng, 1000, 200000), clips=clips,
                     in_place=not clips and rng.random() < 0.5)
    return _clip(None, "layer", 0, 0, 0, 0, d=128 * rng.randint(2, 7), d_ff=128 * rng.randint(4, 38), E=rng.randint(1, 8))


def _tensors(case):
    """(elements, type) of every gradient of a clip case."""
    if case["kind"] == "layer":
        d, f, E = case["d"], case["d_ff"], case["E"]
        return [(d * E, "f32"), (d, "bf16"), (d, "f32")] + [(E * f * d, "f32")] * 3 + [(f * d, "bf16")] * 3
    rng = random.Random(case["sizes_seed"])
    return [(_log_int(rng, case["lo"], case["hi"]), rng.choice(["f32", "bf16"])) for _ in range(case["n"])]


def work(case):
    op = case["op"]
    if op == "clip":
        n_bytes = sum(n * (4 if t == "f32" else 2) for n, t in _tensors(case))
        n_el = sum(n for n, _ in _tensors(case))
        writes = 0 if case["in_place"] else n_bytes       # in place and below the bound nothing has to change
        return {"bytes": n_bytes + writes + 4, "flops": 2 * n_el + (n_el if writes else 0)}
    T, d = case["T"], case["d"]
    if op == "route":
        E, k = case["E"], case["k"]
        b = 2 * T * d + 2 * d * E + 8 * T * k + (4 * E if case["bias"] else 0) + (T if case["mask"] else 0)
        if case["train"]:
            b += 4 * T * E + 8 * E
        return {"bytes": b, "flops": 2 * T * d * E}
    if op == "route_backward":
        E, k = case["E"], case["k"]
        b = 2 * T * d + 2 * d * E + 4 * T * E + 8 * T * k + 4 * T * d + 4 * d * E
        b += (4 * E if case["balance"] else 0) + (T if case["mask"] else 0)
        return {"bytes": b, "flops": 4 * T * d * E}
    e = 2 if case["dtype"] == "bf16" else 4
    n_par = {"none": 0, "rms": 1, "layer": 2}
    params = n_par[case["post"]] + n_par[case["pre"]] + (1 if case["gate"] else 0)
    if op == "norm":
        streams = 3 + (case["pre"] != "none")
        return {"bytes": streams * T * d * e + 2 * params * d, "flops": T * d * (3 + 5 * (case["post"] != "none") + 5 * (case["pre"] != "none"))}
    read = params - (case["pre"] == "layer")               # the shift in front of the next branch has no part in any gradient
    return {"bytes": 6 * T * d * e + 2 * d * read + 4 * d * params, "flops": T * d * (20 + 12 * (case["post"] != "none"))}


# ---------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 17)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _router_inputs(case, g):
    T, d, E = case["T"], case["d"], case["E"]
    x = _randn(g, T, d)
    if case.get("outliers"):
        x[:, torch.randperm(d, generator=g, device="cuda")[:case["outliers"]]] *= 20.0
    w = _randn(g, d, E) * d ** -0.5
    s = {"x": x.to(torch.bfloat16), "w": w.to(torch.bfloat16), "mask": None}
    if case["mask"]:                                   # the last eighth of the batch is padding, and a few tokens inside
        m = torch.rand(T, generator=g, device="cuda") < 0.97
        m[T - T // 8:] = False
        s["mask"] = m.to(torch.uint8)
    return s


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    op = case["op"]
    if op == "route":
        s.update(_router_inputs(case, g))
        s["bias"] = None
        if case["bias"]:
            b = _randn(g, case["E"]) * 0.05
            b[torch.randperm(case["E"], generator=g, device="cuda")[:case["off"]]] = -math.inf
            s["bias"] = b
    elif op == "route_backward":
        s.update(_router_inputs(case, g))
        logits = s["x"].double() @ s["w"].double()
        s["logits"] = logits.float()
        s["idx"] = _plain_select(case, logits)
        if s["mask"] is not None:
            s["idx"][s["mask"] == 0] = -1
        s["d_w"] = _randn(g, case["T"], case["k"]) * 1e-2
        s["d_sum"] = torch.rand(case["E"], generator=g, device="cuda") * 2e-2 if case["balance"] else None
    elif op in ("norm", "norm_backward"):
        T, d, dt = case["T"], case["d"], _dtype(case["dtype"])
        s["r"] = (_randn(g, T, d) * 2.0).to(dt)
        s["y"] = (_randn(g, T, d) * 0.6 + 0.05).to(dt)
        for n in ("post", "pre"):
            s[n + "_gamma"] = (1.0 + 0.2 * _randn(g, d)).to(torch.bfloat16) if case[n] != "none" else None
            s[n + "_beta"] = (0.1 * _randn(g, d)).to(torch.bfloat16) if case[n] == "layer" else None
        s["gate"] = (0.5 + 0.2 * _randn(g, d)).to(torch.bfloat16) if case["gate"] else None
        if op == "norm_backward":
            s["d_total"] = (_randn(g, T, d) * 1e-2).to(dt)
            s["d_normed"] = (_randn(g, T, d) * 1e-2).to(dt)
    else:
        spec = _tensors(case)
        s["grads"] = [(_randn(g, n) * 1e-3).to(_dtype(t)) for n, t in spec]
        s["outs"] = None if case["in_place"] else [torch.empty_like(t) for t in s["grads"]]
        s["max_norm"] = 1e-3 * math.sqrt(sum(n for n, _ in spec)) * (0.5 if case["clips"] else 4.0)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    import paper_2506_14435_amd as M
    case = s["case"]
    if case["op"] == "route":
        s["routing"] = M.MoteRouting(case["k"], score=case["score"], n_groups=case["groups"], top_groups=case["top_groups"],
                                     group_top=case["group_top"], renormalise=case["renorm"], scale=case["scale"])
    elif case["op"] == "route_backward":
        s["routing"] = M.MoteRouting(case["k"], score=case["score"], renormalise=case["renorm"], scale=case["scale"])
    elif case["op"] in ("norm", "norm_backward"):
        side = {n: None if case[n] == "none" else M.MoteNorm(s[n + "_gamma"], s[n + "_beta"], 1e-6) for n in ("post", "pre")}
        s["block"] = M.MoteResidual(case["d"], post=side["post"], gate=s["gate"], pre=side["pre"],
                                    residual_scale=case["residual_scale"], branch_scale=case["branch_scale"])
    else:
        s["clip"] = M.GradClip(s["grads"], s["outs"])


# ------------------------------------------------------------------------------------------------------------- run
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2506_14435_amd as M
    case = s["case"]
    op = case["op"]
    if op == "route":
        r = M.mote_route(s["x"], s["w"], s["routing"], select_bias=s["bias"], token_mask=s["mask"], want_logits=case["train"],
                         want_stats=case["train"])
        return [r.topk_idx, r.topk_w] + ([r.logits, r.counts, r.score_sum] if case["train"] else [])
    if op == "route_backward":
        return list(M.mote_route_backward(s["x"], s["w"], s["routing"], s["logits"], s["idx"], s["d_w"], d_score_sum=s["d_sum"],
                                          token_mask=s["mask"]))
    if op == "norm":
        total, normed = M.mote_residual_norm(s["block"], s["r"], s["y"])
        return [total] if normed is None else [total, normed]
    if op == "norm_backward":
        return [t for t in M.mote_residual_norm_backward(s["block"], s["r"], s["y"], s["d_total"], s["d_normed"]) if t is not None]
    norm = M.mote_clip_grad_norm(s["clip"], s["max_norm"])
    return [norm] + (s["grads"] if s["outs"] is None else s["outs"])


def _plain_select(case, key):
    """The k experts of each row by descending key, ties to the lower index, -1 where none is left."""
    T, E = key.shape
    k, G = case["k"], case.get("groups", 1)
    key = torch.where(torch.isnan(key), torch.full_like(key, torch.finfo(torch.float64).min), key)
    if G > 1:
        per = key.view(T, G, E // G)
        group = torch.sort(per, dim=2, descending=True).values[:, :, :case["group_top"]].sum(2)
        order = torch.sort(group, dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        open_ = torch.zeros(T, G, dtype=torch.bool, device=key.device)
        open_[torch.arange(T, device=key.device)[:, None], order] = True
        key = torch.where(open_[:, :, None], per, torch.full_like(per, -math.inf)).view(T, E)
    top = torch.sort(key, dim=1, descending=True, stable=True)
    idx = top.indices[:, :k]
    return torch.where(top.values[:, :k] == -math.inf, torch.full_like(idx, -1), idx).to(torch.int32)


def _plain_scores(case, logits):
    if case["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-logits))
    e = torch.exp(logits - logits.max(dim=1, keepdim=True).values)
    return e / e.sum(dim=1, keepdim=True)


def _plain_norm(x, gamma, beta):
    if gamma is None:
        return x
    if beta is None:
        return x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + 1e-6) * gamma.float()
    c = x - x.mean(dim=1, keepdim=True)
    return c / torch.sqrt((c * c).mean(dim=1, keepdim=True) + 1e-6) * gamma.float() + beta.float()


def _plain_norm_back(x, gamma, beta, up):
    """Gradients of _plain_norm: (x, gamma, beta)."""
    if gamma is None:
        return up, None, None
    c = x if beta is None else x - x.mean(dim=1, keepdim=True)
    inv = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + 1e-6)
    hat = c * inv
    u = up * gamma.float()
    dx = u - hat * (u * hat).mean(dim=1, keepdim=True)
    if beta is not None:
        dx = dx - u.mean(dim=1, keepdim=True)
    return inv * dx, (up * hat).sum(0), up.sum(0) if beta is not None else None


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "route":
        logits = s["x"].double() @ s["w"].double()          # fp64: neighbouring scores decide indices
        sums = case["groups"] > 1 and case["group_top"] == 2
        key = logits
        if s["bias"] is not None or sums:
            key = _plain_scores(case, logits)
            if s["bias"] is not None:
                key = key + s["bias"].double()
        idx = _plain_select(case, key)
        keep = torch.ones(case["T"], dtype=torch.bool, device=idx.device) if s["mask"] is None else s["mask"] != 0
        idx = torch.where(keep[:, None], idx, torch.full_like(idx, -1))
        l32 = logits.float()
        score = _plain_scores(case, l32)
        at = idx.clamp(min=0).long()
        w = torch.where(idx >= 0, torch.gather(score, 1, at), torch.zeros_like(idx, dtype=torch.float32))
        if case["renorm"]:
            total = w.sum(dim=1, keepdim=True)
            w = torch.where(total > 0, w / total, torch.zeros_like(w))
        w = w * case["scale"]
        if not case["train"]:
            return [idx, w]
        counts = (idx[:, :, None] == torch.arange(case["E"], device=idx.device)).sum(dim=(0, 1)).to(torch.int32)
        return [idx, w, l32, counts, torch.where(keep[:, None], score, torch.zeros_like(score)).sum(0)]
    if op == "route_backward":
        T, E = case["T"], case["E"]
        score = _plain_scores(case, s["logits"])
        chosen = s["idx"] >= 0
        at = s["idx"].clamp(min=0).long()
        up = torch.zeros(T, E, device=score.device).scatter_add_(1, at, torch.where(chosen, s["d_w"], torch.zeros_like(s["d_w"])))
        sel = torch.zeros(T, E, device=score.device).scatter_add_(1, at, chosen.float())
        q = torch.zeros(E, device=score.device) if s["d_sum"] is None else s["d_sum"]
        sigmoid = case["score"] == "sigmoid"
        if case["renorm"]:
            p = score * sel
            p = p / p.sum(dim=1, keepdim=True).clamp(min=1e-38)
            grad = case["scale"] * p * (up - (p * up).sum(dim=1, keepdim=True))
            if sigmoid:
                grad = grad * (1.0 - score) + score * (1.0 - score) * q
            else:
                grad = grad + score * (q - (score * q).sum(dim=1, keepdim=True))
        else:
            up = case["scale"] * up + q
            grad = score * (1.0 - score) * up if sigmoid else score * (up - (score * up).sum(dim=1, keepdim=True))
        if s["mask"] is not None:
            grad = torch.where((s["mask"] != 0)[:, None], grad, torch.zeros_like(grad))
        return [grad @ s["w"].float().t(), s["x"].float().t() @ grad]
    if op in ("norm", "norm_backward"):
        dt = _dtype(case["dtype"])
        r, y = s["r"].float(), s["y"].float()
        a, b = case["residual_scale"], case["branch_scale"]
        z = _plain_norm(y, s["post_gamma"], s["post_beta"])
        gate = 1.0 if s["gate"] is None else s["gate"].float()
        total = a * r + b * (gate * z)
        if op == "norm":
            return [total.to(dt)] + ([] if s["pre_gamma"] is None else [_plain_norm(total, s["pre_gamma"], s["pre_beta"]).to(dt)])
        d_in, d_pre_g, d_pre_b = _plain_norm_back(total, s["pre_gamma"], s["pre_beta"], s["d_normed"].float())
        d_sum = s["d_total"].float() + d_in
        d_z = b * gate * d_sum
        d_gate = None if s["gate"] is None else (b * z * d_sum).sum(0)
        d_y, d_post_g, d_post_b = _plain_norm_back(y, s["post_gamma"], s["post_beta"], d_z)
        return [t for t in ((a * d_sum).to(dt), d_y.to(dt), d_gate, d_post_g, d_post_b, d_pre_g, d_pre_b) if t is not None]
    square = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in s["grads"]:                                      # fp64: a long sum
        square = square + (t.double() * t.double()).sum()
    norm = torch.sqrt(square)
    limit = s["max_norm"]
    coef = torch.where(norm > limit, limit / norm, torch.ones_like(norm)).float()
    if s["outs"] is None:
        for t in s["grads"]:
            t.copy_((t.float() * coef).to(t.dtype))
        outs = s["grads"]
    else:
        outs = [(t.float() * coef).to(t.dtype) for t in s["grads"]]
    return [norm.float().reshape(1)] + list(outs)


# ----------------------------------------------------------------------------------------------------------- exact
def _np64(t):
    return t.detach().double().cpu().numpy()


def _exact_route(case, s):
    x, w = _np64(s["x"]), _np64(s["w"])
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    logits = x @ w
    if case["score"] == "softmax":
        z = np.exp(logits - logits.max(1, keepdims=True))
        score = z / z.sum(1, keepdims=True)
    else:
        score = 1.0 / (1.0 + np.exp(-logits))
    bias = None if s["bias"] is None else _np64(s["bias"])
    key = logits.copy() if bias is None and not (G > 1 and case["group_top"] == 2) else score + (0.0 if bias is None else bias)
    live = np.ones((T, E), dtype=bool)
    if G > 1:
        best = -np.sort(-key.reshape(T, G, E // G), axis=2)[:, :, :case["group_top"]].sum(2)
        rank = np.argsort(-best, axis=1, kind="stable")
        live = np.zeros((T, G), dtype=bool)
        np.put_along_axis(live, rank[:, :case["top_groups"]], True, 1)
        live = np.repeat(live, E // G, axis=1)
    key = np.where(live, key, -np.inf)
    idx = np.argsort(-key, axis=1, kind="stable")[:, :k]
    gone = np.take_along_axis(key, idx, 1) == -np.inf
    keep = np.ones(T, dtype=bool) if s["mask"] is None else s["mask"].cpu().numpy() != 0
    gone |= ~keep[:, None]
    wt = np.where(gone, 0.0, np.take_along_axis(score, idx, 1))
    if case["renorm"]:
        tot = wt.sum(1, keepdims=True)
        wt = np.divide(wt, tot, out=np.zeros_like(wt), where=tot > 0)
    idx = np.where(gone, -1, idx).astype(np.int32)
    out = [torch.from_numpy(idx), torch.from_numpy(wt * case["scale"])]
    if case["train"]:
        counts = np.bincount(idx[idx >= 0], minlength=E).astype(np.int32)
        out += [torch.from_numpy(logits), torch.from_numpy(counts), torch.from_numpy(score[keep].sum(0))]
    return out


def _exact_route_backward(case, s):
    """Differentiates the weights and the score sums by automatic differentiation in fp64."""
    logits = s["logits"].double().requires_grad_(True)
    log_s = torch.log_softmax(logits, dim=1) if case["score"] == "softmax" else torch.nn.functional.logsigmoid(logits)
    there = s["idx"] >= 0
    picked = torch.gather(log_s, 1, s["idx"].clamp(min=0).long())
    if case["renorm"]:
        picked = picked.masked_fill(~there, -math.inf)
        picked = torch.where(there.any(1, keepdim=True), picked, torch.zeros_like(picked))
        wt = torch.softmax(picked, dim=1)
    else:
        wt = picked.exp()
    loss = (torch.where(there, wt, torch.zeros_like(wt)) * s["d_w"].double()).sum() * case["scale"]
    if s["d_sum"] is not None:
        q = log_s.exp() * s["d_sum"].double()
        loss = loss + (q if s["mask"] is None else q * (s["mask"] != 0).double()[:, None]).sum()
    grad, = torch.autograd.grad(loss, logits)
    grad = torch.nan_to_num(grad, nan=0.0)
    return [grad @ s["w"].double().t(), s["x"].double().t() @ grad]


def _exact_norm(case, s):
    leaf = {n: s[n].double().requires_grad_(True) for n in ("r", "y", "gate", "post_gamma", "post_beta", "pre_gamma", "pre_beta")
            if s[n] is not None}

    def norm(v, which):
        if case[which] == "none":
            return v
        if case[which] == "layer":
            v = v - v.mean(1, keepdim=True)
        v = v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt() * leaf[which + "_gamma"]
        return v + leaf[which + "_beta"] if case[which] == "layer" else v

    z = norm(leaf["y"], "post")
    total = case["residual_scale"] * leaf["r"] + case["branch_scale"] * (leaf["gate"] * z if "gate" in leaf else z)
    normed = norm(total, "pre")
    if case["op"] == "norm":
        return [total.detach()] + ([normed.detach()] if case["pre"] != "none" else [])
    names = [n for n in ("r", "y", "gate", "post_gamma", "post_beta", "pre_gamma", "pre_beta") if n in leaf]
    return list(torch.autograd.grad([total, normed], [leaf[n] for n in names], [s["d_total"].double(), s["d_normed"].double()]))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        return _exact_route(case, s)
    if case["op"] == "route_backward":
        return _exact_route_backward(case, s)
    if case["op"] in ("norm", "norm_backward"):
        return _exact_norm(case, s)
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(t, dtype=torch.float64)) ** 2 for t in s["grads"]))
    coef = min(1.0, s["max_norm"] / norm) if norm > 0 else 1.0
    return [torch.tensor([norm], dtype=torch.float64)] + [t.double() * coef for t in s["grads"]]
