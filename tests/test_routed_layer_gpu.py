"""mote_layer_forward_routed on routings with empty slots: they have no row, so nothing that an expert's row could hold reaches their
token, and the experts' work is that of the slots that have one."""
import math

import pytest
import torch

import paper_2506_14435_amd as M
import workloads as W
from tests.mote_testlib import GpuProblem

pytestmark = pytest.mark.gpu


def _routing(T, k, E, seed, empty):
    g = torch.Generator().manual_seed(seed)
    idx = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).to(torch.int32)
    wt = torch.rand(T, k, generator=g)
    idx[torch.rand(T, k, generator=g) < empty] = -1
    return idx.cuda(), wt.cuda()


def _layer_with(gp, alpha):
    t = gp.layer.tensors
    return M.MoteLayer(t["w_router"], t["ws_gate"], t["ws_up"], t["ws_down"], t["wt_gate"], t["wt_up"], t["wt_down"], alpha, gp.layer.top_k)


# plan inside the gate-up kernel, decode tiles, 64-row tiles, 128-row tiles; more than 16 experts
CONFIGS = [W.C1.with_tokens(1, name="one"), W.C1.with_tokens(30, name="thirty"), W.C1.with_tokens(64, name="local"), W.C1.with_tokens(100, name="tiles32"),
           W.C1.with_tokens(700, name="tiles128"), W.MoteConfig("mid", 512, 1024, 16, 2, 400, seed=12), W.MoteConfig("wide", 256, 512, 40, 2, 90, seed=5),
           W.MoteConfig("one_slot", 256, 512, 4, 1, 3000, seed=3)]


@pytest.mark.parametrize("cfg", CONFIGS, ids=lambda c: c.name)
@pytest.mark.parametrize("empty", [0.1, 0.6, 1.0])
def test_empty_slots_have_no_rows(cfg, empty):
    _check_empty_slots(GpuProblem(cfg), empty)


# the kernels that stream wide weights: the plan inside, 32-row tiles, 64-row tiles
@pytest.mark.parametrize("T", [40, 100, 170])
def test_empty_slots_have_no_rows_in_wide_layers(T):
    g = torch.Generator(device="cuda").manual_seed(T)
    d, f = 2048, 8192
    latent = lambda expert, m: torch.randn(*((d, f) if m == 2 else (f, d)), generator=g, device="cuda") * 0.02
    gp = GpuProblem(W.MoteConfig("stream", d, f, 8, 2, T, seed=21), latent_source=latent)
    for empty in (0.2, 1.0):
        _check_empty_slots(gp, empty)


def _check_empty_slots(gp, empty):
    cfg = gp.cfg
    T, k, E = cfg.n_tokens, cfg.top_k, cfg.n_experts
    idx, wt = _routing(T, k, E, cfg.seed + T, empty)
    taps = M.alloc_taps(gp.layer, T, ("topk_idx", "topk_p", "counts", "row_of", "tok_of"))
    got = M.mote_layer_forward_routed(gp.layer, gp.x, idx, wt, taps=taps)
    lean = M.mote_layer_forward_routed(gp.layer, gp.x, idx, wt)
    gone = idx < 0
    want = M.mote_layer_forward_routed(gp.layer, gp.x, torch.where(gone, torch.full_like(idx, E - 1), idx), torch.where(gone, torch.zeros_like(wt), wt))
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(lean, want) and torch.isfinite(got.float()).all()
    n = int((~gone).sum())
    assert torch.equal(taps["counts"].cpu().long(), torch.bincount(idx[~gone].cpu().long(), minlength=E)) and int(taps["counts"].sum()) == n
    assert torch.equal(taps["topk_idx"], idx) and (taps["topk_p"][gone] == 0).all() and (taps["row_of"][gone] == -1).all()
    rows = taps["row_of"][~gone].long()
    assert torch.equal(rows.sort().values.cpu(), torch.arange(n))
    assert torch.equal(taps["tok_of"][rows].long(), torch.arange(T, device="cuda")[:, None].expand(T, k)[~gone])


@pytest.mark.parametrize("cfg", CONFIGS[1:], ids=lambda c: c.name)
def test_an_empty_slot_takes_nothing_from_an_expert_whose_rows_overflow(cfg):
    """Expert 0's scales make its hidden rows infinite; tokens that did not choose it stay finite, whatever slots they leave empty."""
    gp = GpuProblem(cfg)
    T, k, E = cfg.n_tokens, cfg.top_k, cfg.n_experts
    alpha = gp.layer.tensors["alpha"].clone()
    alpha[0] = 3e38
    idx, wt = _routing(T, k, E - 1, cfg.seed, 0.5)
    idx = torch.where(idx >= 0, idx + 1, idx)                                 # nobody chooses expert 0 ...
    plain = M.mote_layer_forward_routed(gp.layer, gp.x, idx, wt)
    got = M.mote_layer_forward_routed(_layer_with(gp, alpha), gp.x, idx, wt)
    torch.cuda.synchronize()
    assert torch.isfinite(plain.float()).all() and torch.equal(got, plain)
    idx[T // 2, 0] = 0                                                        # ... but one token
    got = M.mote_layer_forward_routed(_layer_with(gp, alpha), gp.x, idx, wt)
    torch.cuda.synchronize()
    rest = torch.arange(T, device="cuda") != T // 2
    assert torch.equal(got[rest], plain[rest]) and not torch.isfinite(got[T // 2].float()).all()


@pytest.mark.parametrize("T", [24, 900])
def test_captured_forward_of_routings_that_change(T):
    """A captured call replayed on other routings, of which one is empty and one full."""
    cfg = W.C1.with_tokens(T, name="graph")
    gp = GpuProblem(cfg)
    ws = torch.empty(gp.layer.workspace_bytes(T), dtype=torch.uint8, device="cuda")
    routings = [_routing(T, cfg.top_k, cfg.n_experts, s, e) for s, e in ((1, 0.3), (2, 1.0), (3, 0.0), (4, 0.9))]
    idx, wt = (t.clone() for t in routings[0])
    out = torch.empty_like(gp.x)
    M.mote_layer_forward_routed(gp.layer, gp.x, idx, wt, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mote_layer_forward_routed(gp.layer, gp.x, idx, wt, out=out, workspace=ws)
    for a, b in routings * 2:
        want = M.mote_layer_forward_routed(gp.layer, gp.x, a, b)
        torch.cuda.synchronize()
        idx.copy_(a)
        wt.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
