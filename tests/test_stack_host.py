"""What ResidualNorm, MoEStack and Q8Experts refuse, before any launch (the buffers are host tensors, no GPU is touched)."""
import os

import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import LayerWeights, MoELayer, MoEStack, NormWeights, Q8Experts, ResidualNorm
from paper_2506_02965_amd.synth import LayerConfig

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libpcmoe.so not built")
CFG = LayerConfig("h", T=40, d=128, f=256, E=4, k=2)


def test_stacks_of_unlike_layers():
    one = MoELayer(CFG, device="cpu")
    for other in (dict(T=41), dict(d=256), dict(dtype="f32")):
        with pytest.raises(ValueError, match="share"):
            MoEStack([one, MoELayer(CFG.scaled(**other), device="cpu")])
    with pytest.raises(ValueError, match="twice"):
        MoEStack([one, one])
    with pytest.raises(ValueError, match="needs a layer"):
        MoEStack([])
    with pytest.raises(ValueError, match="pre"):
        MoEStack([one], pre="none")
    with pytest.raises(ValueError, match="not one of"):
        MoEStack([one], post="batch")


def test_shapes_and_types_of_norm_weights(monkeypatch):
    calls = []
    for name in ("moe_residual_norm", "moe_residual_norm_bwd"):
        monkeypatch.setattr(P, name, lambda *a, _n=name, **k: calls.append(_n))
    n = ResidualNorm(40, 128, P.make_norm("rms", "rms", gate_groups=4), device="cpu")
    x = torch.zeros(40, 128, dtype=torch.bfloat16)
    ok = dict(w_post=torch.ones(128).bfloat16(), gate=torch.ones(4, 128).bfloat16(), w_pre=torch.ones(128).bfloat16())
    for name, bad in (("w_post", torch.ones(127).bfloat16()), ("w_pre", torch.ones(128)), ("gate", torch.ones(1, 128).bfloat16()),
                      ("gate", torch.ones(128).bfloat16())):
        with pytest.raises(ValueError, match=name):
            n.forward(NormWeights(**{**ok, name: bad}), x, x)
        with pytest.raises(ValueError, match=name):
            n.backward(NormWeights(**{**ok, name: bad}), x, x)
    for bad in (x[:39], x.float(), x[:, :64]):
        for args in ((bad, x), (x, bad)):
            with pytest.raises(ValueError):
                n.forward(NormWeights(**ok), *args)
            with pytest.raises(ValueError):
                n.backward(NormWeights(**ok), *args)
    assert not calls
    n.forward(NormWeights(**ok), x, x)
    n.backward(NormWeights(**ok), x, x)
    assert calls == ["moe_residual_norm", "moe_residual_norm_bwd"]
    assert n.dgate.shape == (4, 128) and n.dw_pre.dtype == torch.float32


def test_8_bit_experts():
    w = [torch.zeros(2, *s, dtype=torch.float16) for s in ((256, 128), (256, 128), (128, 256))]
    with pytest.raises(ValueError, match="dtype"):
        Q8Experts.pack(LayerWeights(None, None, None, 1, *w))
    q = Q8Experts((None, None), (None, None), (None, None))
    with pytest.raises(ValueError, match="bf16"):
        MoELayer(CFG.scaled(dtype="f32"), device="cpu").forward_q8(LayerWeights(None, None, None, 1, None, None, None), q)


def test_backward_after_forward_q8_is_refused(monkeypatch):
    calls = []
    for name in P.EXPORTS + P.EXPORTS_EXT:
        if name not in ("moe_workspace_size", "moe_status_string", "moe_last_error"):
            monkeypatch.setattr(P, name, lambda *a, _n=name, **k: calls.append(_n), raising=False)
    x = torch.zeros(CFG.T, CFG.d)
    w = LayerWeights(x, None, None, 1, None, None, None)
    layer = MoELayer(CFG, device="cpu")
    layer.forward_q8(w, Q8Experts((None, None), (None, None), (None, None)))
    assert "moe_expert_ffn_q8" in calls
    with pytest.raises(RuntimeError, match="forward_q8"):
        layer.backward(w, x)
    layer.forward(w)
    layer.backward(w, x)
