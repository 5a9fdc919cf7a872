"""What MoEStack hands to the library's calls, recorded in their place (host buffers, no GPU is touched)."""
import os

import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import LayerWeights, MoELayer, MoEStack, NormWeights, Q8Experts, ResidualNorm
from paper_2506_02965_amd.synth import LayerConfig

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libpcmoe.so not built")
CFG = LayerConfig("h", T=64, d=128, f=256, E=4, k=2, n_shared=1)
X_AT = {"moe_route": 1, "moe_permute": 2, "moe_expert_ffn_fwd": 1, "moe_expert_ffn_bwd": 1, "moe_route_bwd": 1}  # x among the arguments


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in P.EXPORTS + P.EXPORTS_EXT:
        if name not in ("moe_workspace_size", "moe_status_string", "moe_last_error"):
            monkeypatch.setattr(P, name, lambda *a, _n=name, **k: made.append((_n, a)), raising=False)
    return made


def weights():
    return LayerWeights(None, None, None, 1, None, None, None)


def stack_of(n, cfg=CFG, **kw):
    return MoEStack([MoELayer(cfg, device="cpu") for _ in range(n)], **kw)


def rows(cfg=CFG):
    return torch.zeros(cfg.T, cfg.d, dtype=torch.bfloat16)


def inputs_of(made):
    """(call, address of its x, rows of x) of every call that reads a layer's input."""
    return [(n, a[X_AT[n]].data_ptr(), a[X_AT[n]].shape[0], a[0].T) for n, a in made if n in X_AT]


def test_backward_reads_this_stacks_inputs_after_another_stacks_forward(calls):
    """Weights shared by two stacks, of 64 tokens and of one, as when a token is decoded between a forward and its backward."""
    one = CFG.scaled(T=1)
    train, decode = stack_of(2), stack_of(2, one)
    ws, ns = [weights(), weights()], [NormWeights()] * 3
    train.forward(rows(), ws, ns)
    decode.forward(rows(one), ws, ns)
    del calls[:]
    train.backward(rows(), ws, ns)
    want = [train.norms[i].h.data_ptr() for i in (1, 1, 0, 0)]
    got = inputs_of(calls)
    assert [g[0] for g in got] == ["moe_expert_ffn_bwd", "moe_route_bwd"] * 2
    assert [g[1] for g in got] == want
    assert all(rows_of_x == T == CFG.T for _, _, rows_of_x, T in got)


def test_layers_with_the_same_weights(calls):
    """Tied layers: each layer's calls read its own input, forward and backward."""
    stack = stack_of(2)
    w = weights()
    ws, ns = [w, w], [NormWeights()] * 3
    stack.forward(rows(), ws, ns)
    first, second = (stack.norms[i].h.data_ptr() for i in range(2))
    assert [g[1] for g in inputs_of(calls)] == [first] * 3 + [second] * 3
    del calls[:]
    stack.backward(rows(), ws, ns)
    assert [g[1] for g in inputs_of(calls)] == [second] * 2 + [first] * 2


def test_weights_norms_and_experts_for_every_layer(calls):
    """As many weights and experts as layers and one norm more, or nothing runs."""
    stack = stack_of(2)
    ws, ns, q = [weights(), weights()], [NormWeights()] * 3, [None] * 2
    for wrong in ((ws[:1], ns, None), (ws + ws, ns, None), (ws, ns[:2], None), (ws, ns + ns, None), (ws, ns, q[:1]), (ws, ns, q + q)):
        with pytest.raises(ValueError, match="layers"):
            stack.forward(rows(), *wrong)
    assert not calls
    stack.forward(rows(), ws, ns)
    del calls[:]
    for wrong in ((ws[:1], ns), (ws + ws, ns), (ws, ns[:2]), (ws, ns + ns)):
        with pytest.raises(ValueError, match="layers"):
            stack.backward(rows(), *wrong)
    assert not calls


def test_layers_that_host_a_part_of_the_experts():
    """Their output is one party's part of a sum, which no norm or residual may take alone."""
    for part in (dict(local_count=2), dict(local_begin=1, local_count=3)):
        layers = [MoELayer(CFG, device="cpu"), MoELayer(CFG.scaled(**part), device="cpu")]
        with pytest.raises(ValueError, match="all experts"):
            MoEStack(layers)
    MoEStack([MoELayer(CFG.scaled(local_count=CFG.E), device="cpu")])


def test_backward_of_what_was_built_without_it(calls):
    stack = MoEStack([MoELayer(CFG, device="cpu"), MoELayer(CFG, device="cpu", backward=False)])
    ws, ns = [weights(), weights()], [NormWeights()] * 3
    stack.forward(rows(), ws, ns)
    norm = ResidualNorm(CFG.T, CFG.d, P.make_norm(), device="cpu", backward=False)
    norm.forward(NormWeights(), rows(), rows())
    del calls[:]
    with pytest.raises(RuntimeError, match="backward=False"):
        stack.backward(rows(), ws, ns)
    with pytest.raises(RuntimeError, match="backward=False"):
        norm.backward(NormWeights(), rows(), rows())
    assert not calls


def test_backward_before_any_forward(calls):
    with pytest.raises(RuntimeError, match="forward"):
        stack_of(1).backward(rows(), [weights()], [NormWeights()] * 2)
    with pytest.raises(RuntimeError, match="forward"):
        ResidualNorm(CFG.T, CFG.d, P.make_norm(), device="cpu").backward(NormWeights(), rows(), rows())
    assert not calls


def test_backward_after_the_layers_ran_elsewhere(calls):
    """A layer holds the activations of its last forward: a backward of an earlier one is refused before anything runs."""
    layers = [MoELayer(CFG, device="cpu") for _ in range(2)]
    first, second = MoEStack(layers), MoEStack(layers, post="rms")
    ws, ns, q = [weights(), weights()], [NormWeights()] * 3, [Q8Experts(*[(None, None)] * 3)] * 2
    others = (lambda: second.forward(rows(), ws, ns), lambda: layers[1].forward(weights()), lambda: layers[0].forward_q8(weights(), q[0]))
    for other in others:
        first.forward(rows(), ws, ns)
        other()
        del calls[:]
        with pytest.raises(RuntimeError, match="forward"):
            first.backward(rows(), ws, ns)
        assert not calls
    second.forward(rows(), ws, ns)
    second.backward(rows(), ws, ns)
    first.forward(rows(), ws, ns, q)
    del calls[:]
    with pytest.raises(RuntimeError, match="forward_q8"):
        first.backward(rows(), ws, ns)
    assert not calls


def test_8_bit_experts_of_another_layer(calls):
    """Codes and scales of other sizes or types than the layer's would be read past their end."""
    G, d, f = CFG.n_groups, CFG.d, CFG.f
    layer = MoELayer(CFG, device="cpu")

    def part(n, rows_, cols, codes=torch.int8, scales=torch.float32):
        return torch.zeros(n, rows_, cols, dtype=codes), torch.zeros(n, rows_, dtype=scales)
    up, down = part(G, f, d), part(G, d, f)
    bad = {"gate": [part(G - 1, f, d), part(G, f // 2, d), part(G, d, f), part(G, f, d, codes=torch.uint8), (up[0], up[1][:, :-1])],
           "up": [part(G, f, 2 * d), part(G, f, d, scales=torch.bfloat16)], "down": [up, (down[0], up[1])]}
    for name, parts in bad.items():
        for p in parts:
            with pytest.raises(ValueError, match=name):
                layer.forward_q8(weights(), Q8Experts(**{**dict(gate=up, up=up, down=down), name: p}))
    assert not calls
    layer.forward_q8(weights(), Q8Experts(up, up, down))
    assert calls
