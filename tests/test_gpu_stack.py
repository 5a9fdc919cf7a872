"""Norms, layers, updates and 8-bit experts together: a stack trained for a few steps and then served.

fp32 gradients of the whole stack are compared with 64-bit autograd at the same routing. Tolerance: every value passes some 40
fp32 products and sums of up to 256 terms in two layers and three norms; relative to the largest gradient of a tensor 2^-24
times 40 times 256 is 6e-4, and twice that is allowed. 8-bit rows are off by a step's half at most: of rows whose largest
magnitude is some 3.5 deviations, 0.8% of a deviation's root mean square for each of x, the weights and H, in a layer's three
products, so that a stack's outputs may be off by a few percent of what the layers add."""
import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import LayerWeights, MoELayer, MoEStack, NormWeights, Q8Experts
from paper_2506_02965_amd.synth import LayerConfig

pytestmark = pytest.mark.gpu


def make(cfg, n, gate_groups, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32

    def normal(*s, std=1.0, mean=0.0):
        return (torch.randn(*s, device="cuda", generator=g) * std + mean).to(dt)
    G, d, f = cfg.n_groups, cfg.d, cfg.f
    ws = [LayerWeights(None, normal(cfg.E, d, std=d ** -0.5), None, 1, normal(G, f, d, std=d ** -0.5),
                       normal(G, f, d, std=d ** -0.5), normal(G, d, f, std=f ** -0.5)) for _ in range(n)]
    ns = [NormWeights(None if i == 0 else normal(d, std=0.1, mean=1.0), None if i == 0 else normal(gate_groups, d, std=0.3, mean=1.0),
                      normal(d, std=0.1, mean=1.0)) for i in range(n + 1)]
    return ws, ns, normal


def stack64(layers, x, ws, ns, eps, alpha, gate_groups, post):
    """The stack in 64 bits at the layers' routing, and its leaves."""
    leaves = {"x": x.double().requires_grad_(True)}
    for i, w in enumerate(ws):
        for k in ("w_router", "w_gate", "w_up", "w_down"):
            leaves[k, i] = getattr(w, k).double().requires_grad_(True)
    for i, n in enumerate(ns):
        for k in ("w_post", "gate", "w_pre"):
            if getattr(n, k) is not None:
                leaves[k, i] = getattr(n, k).double().requires_grad_(True)

    def rms(v, w):
        return v * (v.square().mean(1, keepdim=True) + eps).rsqrt() * w
    r = leaves["x"]
    h = rms(r, leaves["w_pre", 0])
    for i, layer in enumerate(layers):
        idx = layer.topk_idx.long()
        p = torch.softmax((h @ leaves["w_router", i].t()).gather(1, idx), 1)
        y = torch.zeros_like(h)
        for e in range(layer.cfg.E):
            t, j = torch.nonzero(idx == e, as_tuple=True)
            a, u = h[t] @ leaves["w_gate", i][e].t(), h[t] @ leaves["w_up", i][e].t()
            y = y.index_add(0, t, (a * torch.sigmoid(a) * u) @ leaves["w_down", i][e].t() * p[t, j][:, None])
        if post == "rms":
            y = rms(y, leaves["w_post", i + 1])
        g = leaves["gate", i + 1].repeat_interleave(x.shape[0] // gate_groups, 0)
        r = alpha * r + g * y
        h = rms(r, leaves["w_pre", i + 1])
    return h, leaves


def test_gradients_of_a_stack():
    cfg = LayerConfig("s", T=96, d=256, f=128, E=4, k=2, dtype="f32")
    ws, ns, normal = make(cfg, 2, 3)
    layers = [MoELayer(cfg) for _ in range(2)]
    stack = MoEStack(layers, post="rms", residual_scale=0.75, gate_groups=3)
    x, d = normal(cfg.T, cfg.d), normal(cfg.T, cfg.d)
    out = stack.forward(x, ws, ns)
    dx = stack.backward(d, ws, ns)
    want, leaves = stack64(layers, x, ws, ns, float(stack.norms[0].norm.eps), 0.75, 3, "rms")
    names = list(leaves)
    grads = dict(zip(names, torch.autograd.grad(want, [leaves[k] for k in names], d.double())))
    tol = 2 * 40 * 256 * 2.0 ** -24

    def close(a, b, what):
        off = float((a.double() - b).abs().max() / b.abs().max())
        assert off <= tol, (what, off)
    close(out, want.detach(), "out")
    close(dx, grads["x"], "x")
    for i, layer in enumerate(layers):
        for k in ("gate", "up", "down"):
            close(getattr(layer, "dw_" + k), grads["w_" + k, i], (k, i))
        close(layer.dw_router, grads["w_router", i], ("router", i))
    for i, n in enumerate(stack.norms):
        close(n.dw_pre, grads["w_pre", i], ("w_pre", i))
        if i:
            close(n.dw_post, grads["w_post", i], ("w_post", i))
            close(n.dgate, grads["gate", i], ("gate", i))


@pytest.mark.parametrize("final", ["rms", "none"])
def test_train_update_and_serve(final):
    cfg = LayerConfig("s", T=128, d=256, f=384, E=8, k=2, n_shared=1)
    ws, ns, normal = make(cfg, 2, 1, seed=3)
    layers = [MoELayer(cfg) for _ in range(2)]
    stack = MoEStack(layers, post="rms", final=final, gate_groups=1)
    if final == "none":
        ns[-1].w_pre = None
    for layer, w in zip(layers, ws):
        layer.init_muon_state(w)
    opt = P.make_muon(lr=1e-3, scale=0.2 * cfg.f ** 0.5, weight_decay=0.01)
    x, target = normal(cfg.T, cfg.d), normal(cfg.T, cfg.d)
    for _ in range(3):
        out = stack.forward(x, ws, ns)
        d = ((out.float() - target.float()) / cfg.T).bfloat16()
        before = [w.w_up.clone() for w in ws]
        stack.backward(d, ws, ns)
        for i, (layer, w) in enumerate(zip(layers, ws)):
            layer.update_muon(w, opt)
            step = (w.w_up.float() - before[i].float()).pow(2).mean().sqrt()
            # the update's elements have an rms of some 0.2 lr (the polynomial leaves singular values around 1)
            assert 0.3 * 0.2e-3 < float(step) < 3 * 0.2e-3
            assert torch.equal(w.w_up.reshape(-1), layer.muon_master[w.w_gate.numel():2 * w.w_gate.numel()].bfloat16())
    out = stack.forward(x, ws, ns).clone()
    r = stack.norms[-1].r.clone()
    q = [Q8Experts.pack(w) for w in ws]
    small = stack.forward(x, ws, ns, q)
    added = (r.float() - x.float()).norm()
    assert float((stack.norms[-1].r.float() - r.float()).norm() / added) < 0.1
    assert torch.isfinite(small.float()).all()
    with pytest.raises(RuntimeError, match="forward_q8"):
        stack.backward(out, ws, ns)
    # a prompt's tokens one at a time, through the same weights
    one = LayerConfig("t", T=1, d=256, f=384, E=8, k=2, n_shared=1, backward=False)
    token = MoEStack([MoELayer(one) for _ in range(2)], post="rms", final=final, gate_groups=1)
    for t in (0, 77):
        got = token.forward(x[t:t + 1].contiguous(), ws, ns, q)
        # routing is decided on sums whose order follows the batch's size: the same experts but for ties, the same codes
        assert float((got.float() - small[t:t + 1].float()).norm() / small[t:t + 1].float().norm()) < 0.02


def test_the_examples_prompt():
    """The example's prompt through 8-bit experts. x, H and the weights are off by some 1% of a row's size each; tokens for which
    two experts are nearly equal may take the other."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import gated_experts as G
    student, _ = G.train(2, 64, log=lambda *a: None)
    assert G.prompt(student, 130, log=lambda *a: None) < 0.2


def test_a_captured_training_step():
    cfg = LayerConfig("s", T=64, d=128, f=256, E=4, k=2)
    ws, ns, normal = make(cfg, 2, 2, seed=5)
    layers = [MoELayer(cfg) for _ in range(2)]
    stack = MoEStack(layers, gate_groups=2)
    for n in ns:
        n.w_post = None
    for layer, w in zip(layers, ws):
        layer.init_muon_state(w, master=False)
    opt = P.make_muon(lr=1e-3)
    x, d = normal(cfg.T, cfg.d), normal(cfg.T, cfg.d)

    def step():
        out = stack.forward(x, ws, ns)
        dx = stack.backward(d, ws, ns)
        for layer, w in zip(layers, ws):
            layer.update_muon(w, opt)
        return out, dx
    state = [t for w in ws for t in (w.w_gate, w.w_up, w.w_down)] + [l.muon_m for l in layers]
    step()                                         # buffers of the first call
    start = [t.clone() for t in state]
    eager = []
    for _ in range(3):
        out, dx = step()
        eager.append([t.clone() for t in (out, dx, *state)])
    for t, s in zip(state, start):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out, dx = step()
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, dx, *state), want))


def test_a_backward_after_another_stacks_forward():
    """Two stacks with the same weights: the first one's gradients are those that it gives alone."""
    cfg = LayerConfig("s", T=96, d=256, f=128, E=4, k=2, n_shared=1)
    ws, ns, normal = make(cfg, 2, 1, seed=7)
    first, second = (MoEStack([MoELayer(c) for _ in range(2)]) for c in (cfg, cfg.scaled(T=33)))
    for n in ns:
        n.w_post = None
    x, other, d = normal(cfg.T, cfg.d), normal(33, cfg.d), normal(cfg.T, cfg.d)

    def gradients(between):
        first.forward(x, ws, ns)
        if between:
            second.forward(other, ws, ns)
        dx = first.backward(d, ws, ns)
        return [t.clone() for l in first.layers for t in (l.dw_gate, l.dw_up, l.dw_down, l.dw_router)] + [dx.clone()]
    alone = gradients(False)
    assert all(torch.equal(a, b) for a, b in zip(alone, gradients(True)))
