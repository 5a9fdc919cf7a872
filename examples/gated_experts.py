"""Two expert layers trained and then served, on one GPU:

    python examples/gated_experts.py [--steps 60] [--tokens 512]

Training: gated routing (sigmoid scores, limited expert groups, a balance bias that follows the experts' load), the layers'
activations kept in 8 bits between forward and backward, with one full-size buffer for both layers, and AdamW on the experts.
The stack x -> x + layer(x) learns to imitate a fixed random one. Serving: the trained experts packed to 4 bits, tokens one at
a time, compared with the bf16 layers. All steps of the layers run in the library's kernels.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_02965_amd import pcmoe as P  # noqa: E402
from paper_2506_02965_amd.layer import LayerWeights, MoELayer, Q4Experts  # noqa: E402
from paper_2506_02965_amd.synth import LayerConfig  # noqa: E402

LAYERS = 2


def config(tokens, backward=True):
    return LayerConfig("example", T=tokens, d=512, f=1024, E=32, k=4, n_shared=1, backward=backward)


def gate():
    return P.make_gate("sigmoid", n_groups=8, topk_groups=4, group_top=2, scale=1.0)


def weights(cfg, gen):
    def normal(*shape, std):
        return (torch.randn(*shape, device="cuda", generator=gen) * std).bfloat16()
    G, d, f = cfg.n_groups, cfg.d, cfg.f
    return LayerWeights(torch.empty(cfg.T, d, device="cuda", dtype=torch.bfloat16), normal(cfg.E, d, std=d ** -0.5), None, 1,
                        normal(G, f, d, std=d ** -0.5), normal(G, f, d, std=d ** -0.5), normal(G, d, f, std=f ** -0.5),
                        select_bias=torch.zeros(cfg.E, device="cuda"))


def stack_forward(layers, ws, x):
    """x -> x + layer(x), layer by layer; each layer's input stays in its weights' `x` for the backward."""
    for layer, w in zip(layers, ws):
        w.x = x
        x = x + layer.forward(w)
    return x


def train(steps, tokens, log=print):
    cfg = config(tokens)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    teacher = [weights(cfg, gen) for _ in range(LAYERS)]
    student = [weights(cfg, gen) for _ in range(LAYERS)]
    shared = torch.empty(P.moe_workspace_size(MoELayer(cfg, backward=False).desc, P.MOE_WS_FFN_SAVED), dtype=torch.uint8,
                         device="cuda")
    layers = [MoELayer(cfg, gate=gate(), checkpoint=True, saved=shared) for _ in range(LAYERS)]
    truth = [MoELayer(cfg, backward=False, gate=gate()) for _ in range(LAYERS)]
    for layer, w in zip(layers, student):
        layer.init_update_state(w)
    routers = [w.w_router.float() for w in student]
    losses = []
    for step in range(steps):
        x = torch.randn(cfg.T, cfg.d, device="cuda", generator=gen).bfloat16()
        target = stack_forward(truth, teacher, x)
        diff = (stack_forward(layers, student, x) - target).float()
        losses.append(float(diff.square().mean()))
        dy = (diff * (2.0 / cfg.T)).bfloat16()
        for i in reversed(range(LAYERS)):
            layer, w = layers[i], student[i]
            dy = dy + layer.backward(w, dy)
            layer.update(w, P.make_opt("adamw", lr=1e-3))
            routers[i] -= 1e-2 * layer.dw_router
            w.w_router = routers[i].bfloat16()
            load = layer.counts.float()
            w.select_bias += 1e-3 * torch.sign(load.mean() - load)     # more load for the experts that have too little
        if step % 10 == 0 or step == steps - 1:
            load = layers[0].counts.float()
            log(f"step {step:3d}  loss {losses[-1]:.4f}  busiest expert {float(load.max() / load.mean()):.2f} x the mean load")
    full = layers[0].saved.numel()
    log(f"saved for the backward: {LAYERS} checkpoints of {layers[0].ckpt.numel() / 1e6:.1f} MB and one buffer of "
        f"{full / 1e6:.1f} MB, in place of {LAYERS} such buffers")
    return student, losses


def serve(student, tokens=16, log=print):
    cfg = config(1, backward=False)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    packed = [Q4Experts.pack(w, 64) for w in student]
    exact = [MoELayer(cfg, gate=gate()) for _ in range(LAYERS)]
    small = [MoELayer(cfg, gate=gate()) for _ in range(LAYERS)]
    off = norm = 0.0
    for _ in range(tokens):
        x = torch.randn(1, cfg.d, device="cuda", generator=gen).bfloat16()
        y = x
        for layer, w, q in zip(small, student, packed):
            w.x = y
            y = y + layer.forward_q4(w, q)
        ref = stack_forward(exact, student, x)
        off += float((y - ref).float().square().sum())
        norm += float((ref - x).float().square().sum())
    rel = (off / norm) ** 0.5
    bits = 8 * sum(t.numel() * t.element_size() for q in packed for p in (q.gate, q.up, q.down) for t in p)
    params = sum(t.numel() for w in student for t in (w.w_gate, w.w_up, w.w_down))
    log(f"{tokens} tokens with {bits / params:.2f}-bit experts: {100 * rel:.1f}% off what the bf16 layers add to them")
    return rel


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=512)
    a = ap.parse_args()
    student, _ = train(a.steps, a.tokens)
    serve(student)


if __name__ == "__main__":
    main()
