"""Gated routing and its adjoint against their definitions in 64 bits, evaluated on the CPU.

Selection is compared exactly, on the fp32 scores that the call returned. A gate weight is an fp64 value rounded once to
fp32: within 2^-23 of it (half an ulp, and as much again for the exponentials)."""
import math

import numpy as np
import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import MoELayer, upload
from paper_2506_02965_amd.synth import LayerConfig, make_inputs
from gpu_util import check_logits, log

pytestmark = pytest.mark.gpu


def select(l, bias, k, score, groups, keep, top, renorm, scale):
    """Token by token in numpy fp64: (idx, w)."""
    T, E = l.shape
    idx = np.full((T, k), P.MOE_NO_EXPERT, np.int64)
    w = np.zeros((T, k))
    n = E // groups
    for t in range(T):
        ok = l[t] > -np.inf
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                s = 1 / (1 + np.exp(-l[t]))
        elif ok.any():
            m = l[t][ok].max()
            s = np.where(ok, np.exp(np.where(ok, l[t] - m, 0)), 0)
            s = s / s.sum()
        else:
            s = np.zeros(E)
        if bias is None:
            key, value = l[t], (s if top == 2 else l[t])
        else:
            key = value = s + bias
            ok = ok & (bias > -np.inf)
        chosen = [e for e in range(E) if ok[e]]
        if groups > 1:
            worth = []
            for g in range(groups):
                v = sorted((value[e] for e in range(g * n, g * n + n) if ok[e]), reverse=True)[:top]
                worth.append(sum(v) if v else -math.inf)
            kept = sorted(range(groups), key=lambda g: (-worth[g], g))[:keep]
            chosen = [e for e in chosen if e // n in kept]
        chosen = sorted(chosen, key=lambda e: (-key[e], e))[:k]
        idx[t, :len(chosen)] = chosen
        v = s[chosen]
        if renorm and len(chosen):
            if score == "softmax":
                v = np.exp(l[t][chosen] - l[t][chosen].max())
            v = v / v.sum() if v.sum() > 0 else 0 * v
        w[t, :len(chosen)] = v * scale
    return idx, w


def route(T, d, E, k, dtype, gate, renorm, bias=None, logit_bias=None, edit=None, seed=3):
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn(T, d, generator=gen).to(dt)
    wr = (torch.randn(E, d, generator=gen) * d ** -0.5).to(dt)
    if edit:
        edit(x, wr)
    desc = P.make_desc(T, d, 128, E, k, renormalize=renorm, dtype=dtype)
    logits = torch.full((T, E), 7.0, device="cuda")
    idx = torch.full((T, k), -3, dtype=torch.int32, device="cuda")
    gw = torch.full((T, k), -3.0, device="cuda")
    up = lambda t: None if t is None else t.cuda()
    P.moe_route_gated(desc, gate, x.cuda(), wr.cuda(), up(logit_bias), 1 if logit_bias is None else logit_bias.shape[0],
                      up(bias), logits, idx, gw)
    torch.cuda.synchronize()
    s = x.double() @ wr.double().t()
    if logit_bias is not None:
        s = s + logit_bias.double().repeat_interleave(T // logit_bias.shape[0], 0)
    return s, logits.cpu(), idx.cpu(), gw.cpu(), desc, x, wr


def check(logits, idx, gw, bias, k, g, renorm):
    score = "sigmoid" if g["score"] == "sigmoid" else "softmax"
    ri, rw = select(logits.double().numpy(), None if bias is None else bias.double().numpy(), k, score,
                    g.get("n_groups", 1), g.get("topk_groups", 1), g.get("group_top", 1), renorm, g.get("scale", 1.0))
    assert np.array_equal(idx.long().numpy(), ri), "topk_idx differs"
    err = np.abs(gw.double().numpy() - rw)
    assert np.all(err <= 2.0 ** -23 * np.abs(rw) + 1e-44), err.max()


CASES = [  # T, d, E, k, groups, keep, top
    (1, 128, 4, 2, 1, 1, 1), (3, 256, 16, 1, 4, 2, 1), (257, 384, 16, 3, 2, 1, 2), (255, 256, 64, 6, 8, 4, 2),
    (1025, 128, 65, 4, 5, 2, 2), (300, 256, 256, 8, 8, 4, 2), (2000, 128, 200, 8, 25, 3, 2), (4097, 128, 256, 8, 64, 2, 1),
    (4100, 128, 32, 2, 16, 16, 2), (33, 128, 96, 8, 3, 3, 1), (8195, 128, 40, 6, 20, 3, 2), (700, 128, 33, 8, 1, 1, 2),
    (40, 128, 8, 8, 1, 1, 1), (64, 128, 256, 4, 2, 1, 2),
    # the scores spread over the CUs, 16, 32 and 64 experts to a workgroup of 1, 4, 16 and 32 tokens
    (1, 1024, 64, 6, 8, 4, 2), (3, 512, 200, 8, 1, 1, 1), (62, 768, 66, 4, 2, 2, 1), (150, 512, 100, 3, 5, 2, 2),
    (300, 1024, 50, 2, 1, 1, 1), (501, 384, 129, 8, 3, 2, 2), (999, 256, 199, 4, 1, 1, 1), (2047, 256, 256, 8, 16, 4, 2),
    (1050, 768, 64, 6, 1, 1, 1),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "T{}_d{}_E{}_k{}_g{}_{}_{}".format(*c))
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
def test_selection(case, score, with_bias):
    T, d, E, k, groups, keep, top = case
    renorm, dtype = (T + k) % 2 == 0, "f32" if E % 3 == 0 else "bf16"
    g = dict(score=score, n_groups=groups, topk_groups=keep, group_top=top, scale=2.5 if T % 2 else 1.0)
    gen = torch.Generator().manual_seed(T)
    bias = (torch.randn(E, generator=gen) * 30).round() * 0.001 if with_bias else None
    lb = torch.randn(1, E, generator=gen) if T % 3 == 0 else None
    log(f"[gated] {case} {score} bias={with_bias} {dtype} renormalize={renorm}")
    s, logits, idx, gw, *_ = route(T, d, E, k, dtype, P.make_gate(**g), renorm, bias, lb)
    check_logits(logits, s.float().numpy())
    check(logits, idx, gw, bias, k, g, renorm)


@pytest.mark.parametrize("T", [5, 500, 5000])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_masks_ties_and_special_scores(T, score, renorm):
    """Per-party masks of -inf that leave all, one, two or no experts, the lowest fp32 number, NaN scores, biases of NaN, -inf
    and +inf, duplicated experts (ties within and between groups), scores far apart."""
    E, k = 24, 4
    lb = torch.zeros(5, E)
    lb[1, 3:] = -math.inf                       # three experts of the first group
    lb[2] = -math.inf                           # nothing
    lb[3, 1:] = torch.finfo(torch.float32).min  # selectable, but for softmax without weight
    lb[4, ::2] = -math.inf
    lb[4, 5] = math.nan

    def edit(x, wr):
        wr[6:12] = wr[0:6]
        x[-1] = 0            # every score 0
        if x.shape[0] > 4:
            x[0] *= 100      # scores far apart

    for bias_kind in ("none", "plain", "special"):
        bias = None
        if bias_kind != "none":
            bias = torch.zeros(E)
            bias[7] = 0.25
        if bias_kind == "special":
            bias[9], bias[10], bias[13], bias[20] = -math.inf, math.nan, math.inf, -0.0
        for groups, keep, top in ((1, 1, 1), (4, 2, 2), (4, 2, 1), (12, 3, 2)):
            g = dict(score=score, n_groups=groups, topk_groups=keep, group_top=top)
            log(f"[gated] special T={T} {score} renormalize={renorm} bias={bias_kind} groups={groups}/{keep} top={top}")
            _, logits, idx, gw, *_ = route(T, 128, E, k, "f32", P.make_gate(**g), renorm, bias, lb, edit)
            check(logits, idx, gw, bias, k, g, renorm)
            per = T // 5
            assert bool((idx[2 * per:3 * per] == P.MOE_NO_EXPERT).all()) and not gw[2 * per:3 * per].any()


@pytest.mark.parametrize("renorm", [False, True])
def test_plain_softmax_is_the_ungated_routing(renorm):
    T, d, E, k = 777, 256, 64, 6
    s, logits, idx, gw, desc, x, wr = route(T, d, E, k, "bf16", P.make_gate(), renorm)
    lg, i2, w2 = torch.empty(T, E, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda"), \
        torch.empty(T, k, device="cuda")
    P.moe_route(desc, x.cuda(), wr.cuda(), None, 1, lg, i2, w2)
    assert torch.equal(lg.cpu(), logits) and torch.equal(i2.cpu(), idx)
    assert float(((w2.cpu() - gw).abs() / gw).max()) <= 1e-6      # fp32 exponentials there


def gate_formula(l, idx, g, w, score, renorm, scale):
    """dlogits in fp64 torch from the returned weights."""
    ok = idx < l.shape[1]
    at = torch.where(ok, idx, 0)
    w, g = torch.where(ok, w, 0), torch.where(ok, g, 0)
    dl = torch.zeros_like(l)
    if score == "softmax" and not renorm:
        m = l > -math.inf
        e = torch.where(m, torch.exp(l - torch.where(m, l, -math.inf).amax(1, keepdim=True).clamp(min=-1e308)), 0)
        z = e.sum(1, keepdim=True)
        p = torch.where(z > 0, e / z, 0)
        gd = torch.zeros_like(l).scatter_add_(1, at, torch.where(ok, scale * g, 0))
        return p * (gd - (p * gd).sum(1, keepdim=True))
    v = w * (g - (w * g).sum(1, keepdim=True) / scale) if renorm else w * g
    if score == "sigmoid":
        v = v * torch.sigmoid(-l.gather(1, at))
    return dl.scatter_add_(1, at, torch.where(ok, v, 0))


GRADS = [(1, 128, 4, 2), (2, 128, 256, 8), (31, 256, 8, 1), (33, 128, 64, 6), (257, 128, 17, 8), (1500, 512, 8, 2),
         (700, 128, 200, 8), (3000, 256, 96, 4), (4096, 128, 256, 8), (258, 128, 66, 3), (1000, 256, 33, 2), (34, 640, 12, 4),
         (16384, 128, 64, 6), (4098, 256, 130, 8), (514, 384, 17, 2), (8200, 4096, 24, 2)]


@pytest.mark.parametrize("case", GRADS, ids=lambda c: "T{}_d{}_E{}_k{}".format(*c))
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient(case, score, renorm):
    """Against the formula from the same inputs in fp64. A score's gradient is some ten fp32 operations, of which the
    differences cancel: within 32 * 2^-24 of the token's largest term; the weight's: sums of T such products, within
    2e-6 of the norm (an fp32 sum of a few hundred terms and a sum over chunks)."""
    T, d, E, k = case
    dtype, scale = "f32" if T % 2 else "bf16", 2.5 if k > 2 else 1.0
    gen = torch.Generator().manual_seed(T + E)
    lb = torch.zeros(1, E)
    if T == 33:
        lb[:, 2:] = -math.inf      # two experts left: slots that none fills
    gate = P.make_gate(score, scale=scale)
    log(f"[gated grad] {case} {score} renormalize={renorm} {dtype}")
    _, logits, idx, gw, desc, x, wr = route(T, d, E, k, dtype, gate, renorm, None, lb)
    g = torch.randn(T, k, generator=gen)
    if T == 33:
        assert bool((idx[:, 2:] == P.MOE_NO_EXPERT).all())
        g[:, 2:] = math.nan        # what stands in an empty slot's gradient does not count
    dl, dw = torch.full((T, E), 9.0, device="cuda"), torch.full((E, d), 9.0, device="cuda")
    ws = torch.empty(max(1, P.moe_workspace_size(desc, P.MOE_WS_ROUTE_BWD)), dtype=torch.uint8, device="cuda")
    P.moe_route_gated_bwd(desc, gate, x.cuda(), logits.cuda(), idx.cuda(), gw.cuda(), g.cuda(), dl, dw, ws, ws.numel())
    torch.cuda.synchronize()
    ref = gate_formula(logits.double(), idx.long(), g.double(), gw.double(), score, renorm, scale)
    size = (gw.double() * torch.nan_to_num(g.double())).abs().amax(1, keepdim=True) + 1e-30
    assert float(((dl.cpu().double() - ref).abs() / size).max()) <= 32 * 2.0 ** -24
    dwr = ref.t() @ x.double()
    assert float((dw.cpu().double() - dwr).norm() / (dwr.norm() + 1e-30)) <= 2e-6 or float(dwr.norm()) == 0.0


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(score, renorm):
    """<g, w> as a function of the scores, selection held: central differences in fp64, step 1e-5 (error about 1e-10), for
    the gradients that the call forms in fp32 (2^-20 of the largest)."""
    T, d, E, k, scale = 6, 128, 12, 3, 2.0
    gate = P.make_gate(score, 3, 2, 2, scale)
    _, logits, idx, gw, desc, x, _ = route(T, d, E, k, "f32", gate, renorm)
    g = torch.randn(T, k, generator=torch.Generator().manual_seed(1))
    dl, dw = torch.empty(T, E, device="cuda"), torch.empty(E, d, device="cuda")
    ws = torch.empty(max(1, P.moe_workspace_size(desc, P.MOE_WS_ROUTE_BWD)), dtype=torch.uint8, device="cuda")
    P.moe_route_gated_bwd(desc, gate, x.cuda(), logits.cuda(), idx.cuda(), gw.cuda(), g.cuda(), dl, dw, ws, ws.numel())
    torch.cuda.synchronize()

    def value(l):
        s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, 1)
        w = s.gather(1, idx.long())
        return float(((w / w.sum(1, keepdim=True) if renorm else w) * scale * g.double()).sum())

    l = logits.double()
    num = torch.zeros_like(l)
    for t in range(T):
        for e in range(E):
            h = torch.zeros_like(l)
            h[t, e] = 1e-5
            num[t, e] = (value(l + h) - value(l - h)) / 2e-5
    assert float((dl.cpu().double() - num).abs().max() / num.abs().max()) <= 2.0 ** -20


def test_layer_with_empty_slots():
    """A whole layer step whose mask leaves some tokens without an expert: their outputs and gradients are zeros, and the
    other tokens' are those of a batch without them."""
    cfg = LayerConfig("g", T=64, d=256, f=256, E=8, k=2, seed=3)
    inp = make_inputs(cfg, with_dy=True)
    w = upload(inp)
    lb = torch.zeros(64, 8, device="cuda")
    lb[5], lb[40] = -math.inf, -math.inf
    w.logit_bias, w.bias_groups = lb, 64
    w.select_bias = torch.linspace(-0.01, 0.01, 8, device="cuda")
    layer = MoELayer(cfg, gate=P.make_gate("sigmoid", 4, 2, 2, 1.5))
    layer.forward(w)
    layer.backward(w)
    torch.cuda.synchronize()
    none = torch.tensor([5, 40], device="cuda")
    assert not layer.y[none].any() and not layer.dx[none].any() and not layer.dlogits[none].any()
    assert int(layer.offsets[-1]) == 62 * 2
    keep = torch.ones(64, dtype=torch.bool, device="cuda")
    keep[none] = False
    sub = cfg.scaled(T=62)
    w2 = upload(inp)
    w2.x, w2.dy, w2.select_bias = w.x[keep].contiguous(), w.dy[keep].contiguous(), w.select_bias
    other = MoELayer(sub, gate=P.make_gate("sigmoid", 4, 2, 2, 1.5))
    other.forward(w2)
    other.backward(w2)
    torch.cuda.synchronize()
    assert torch.equal(other.topk_idx, layer.topk_idx[keep])
    for a, b in ((layer.y[keep], other.y), (layer.dx[keep], other.dx)):
        assert float((a.float() - b.float()).abs().max() / b.float().abs().max()) <= 2e-2


def test_training_step_graph_replays():
    """Forward and backward with gated routing and 8-bit checkpoints captured into a graph: replays on other inputs, with eager
    work in between, equal the eager step bit for bit."""
    cfg = LayerConfig("gt", T=300, d=256, f=384, E=64, k=4, n_shared=1, seed=12)
    inp = make_inputs(cfg, with_dy=True)
    w = upload(inp)
    w.select_bias = torch.linspace(-0.02, 0.02, 64, device="cuda")
    gate = P.make_gate("sigmoid", 8, 4, 2, 2.0)
    layer, eager = MoELayer(cfg, gate=gate, checkpoint=True), MoELayer(cfg, gate=gate, checkpoint=True)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        layer.forward(w)
        layer.backward(w)
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        layer.forward(w)
        layer.backward(w)
    for seed in range(4):
        w.x.copy_(torch.randn(300, 256, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        eager.forward(w)
        eager.backward(w)
        torch.cuda.synchronize()
        for name in ("y", "dx", "dw_gate", "dw_up", "dw_down", "dw_router", "dlogits", "topk_idx"):
            assert torch.equal(getattr(layer, name), getattr(eager, name)), (seed, name)
