"""What MoELayer and Q4Experts refuse, before any launch (no GPU is touched: the layers' buffers are host tensors)."""
import os

import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import LayerWeights, MoELayer, Q4Experts, training_footprint
from paper_2506_02965_amd.synth import LayerConfig

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libpcmoe.so not built")
CFG = LayerConfig("h", T=40, d=128, f=256, E=4, k=2, n_shared=1)


def saved_bytes(cfg):
    return P.moe_workspace_size(MoELayer(cfg, device="cpu", backward=False).desc, P.MOE_WS_FFN_SAVED)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_buffer_of_a_smaller_layer_is_refused(dtype):
    cfg = CFG.scaled(dtype=dtype)
    need = saved_bytes(cfg)
    for n in (0, 1, need - 1, saved_bytes(cfg.scaled(T=39)), saved_bytes(cfg.scaled(f=128))):
        with pytest.raises(ValueError, match=f"{need} bytes"):
            MoELayer(cfg, device="cpu", checkpoint=True, saved=torch.empty(n, dtype=torch.uint8))
    for ok in (torch.empty(need, dtype=torch.uint8), torch.empty(saved_bytes(cfg.scaled(T=41)), dtype=torch.uint8),
               torch.empty((need + 3) // 4, dtype=torch.float32)):
        assert MoELayer(cfg, device="cpu", checkpoint=True, saved=ok).saved is ok


def test_shared_buffer_elsewhere_or_strided_is_refused():
    need = saved_bytes(CFG)
    with pytest.raises(ValueError, match="device"):
        MoELayer(CFG, device="cpu", checkpoint=True, saved=torch.empty(need, dtype=torch.uint8, device="meta"))
    with pytest.raises(ValueError, match="contiguous"):
        MoELayer(CFG, device="cpu", checkpoint=True, saved=torch.empty(2 * need, dtype=torch.uint8)[::2])


@pytest.mark.parametrize("dtype", ["fp16", "bfloat16", "half", "", None])
def test_weight_types_other_than_the_librarys_are_refused(dtype):
    """Read as fp32, a 16-bit tensor would be read past its end."""
    for call in (P.moe_q4_pack, P.moe_q4_unpack):
        with pytest.raises(ValueError, match="dtype"):
            call(1, 16, 128, 32, dtype, None, None, None, stream=0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_packing_other_weight_types_is_refused(dtype):
    w = [torch.zeros(2, *s, dtype=dtype) for s in ((256, 128), (256, 128), (128, 256))]
    with pytest.raises(ValueError, match="dtype"):
        Q4Experts.pack(LayerWeights(None, None, None, 1, *w))


def test_backward_needs_the_activations_of_its_own_forward(monkeypatch):
    """forward_q4 routes anew and saves nothing: a backward after it would read activations (or, where no forward ran, a tile
    plan) that do not belong to its rows."""
    calls = []
    for name in P.EXPORTS + P.EXPORTS_EXT:
        if name not in ("moe_workspace_size", "moe_status_string", "moe_last_error"):
            monkeypatch.setattr(P, name, lambda *a, _n=name, **k: calls.append(_n), raising=False)
    x = torch.zeros(CFG.T, CFG.d)
    w = LayerWeights(x, None, None, 1, None, None, None)
    q = Q4Experts(32, (None, None), (None, None), (None, None))
    for checkpoint in (False, True):
        layer = MoELayer(CFG, device="cpu", checkpoint=checkpoint)
        layer.forward_q4(w, q)
        calls.clear()
        with pytest.raises(RuntimeError, match="forward_q4"):
            layer.backward(w, x)
        assert not calls
        layer.forward(w)
        layer.backward(w, x)
        assert "moe_expert_ffn_bwd" in calls
        layer.forward_q4(w, q)
        with pytest.raises(RuntimeError, match="forward_q4"):
            layer.ffn_bwd(w, x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_footprint_of_a_checkpointed_layer(dtype):
    """What a layer with checkpoint=True allocates, its own saved buffer or one that several layers share: the accounts differ
    by the buffers that MoELayer allocates."""
    cfg = CFG.scaled(dtype=dtype)
    plain = training_footprint(cfg, cfg.E)
    desc = MoELayer(cfg, device="cpu", backward=False).desc
    saved, ckpt = (P.moe_workspace_size(desc, which) for which in (P.MOE_WS_FFN_SAVED, P.MOE_WS_FFN_CKPT))
    own = MoELayer(cfg, device="cpu", backward=False, checkpoint=True)
    assert (own.saved.numel(), own.ckpt.numel()) == (saved, ckpt)
    one = training_footprint(cfg, cfg.E, checkpoint=True)
    assert one["activations"] == plain["activations"] + ckpt and one["total"] == plain["total"] + ckpt
    shared = training_footprint(cfg, cfg.E, checkpoint=True, shared_saved=True)
    assert shared["activations"] == plain["activations"] - saved + ckpt
    assert shared["total"] == plain["total"] - saved + ckpt and shared["shared_saved"] == saved
    assert {k: v for k, v in training_footprint(cfg, cfg.E, checkpoint=False).items()} == plain
    with pytest.raises(ValueError):
        training_footprint(cfg, cfg.E, shared_saved=True)


def test_current_stream_without_torchs_private_names(monkeypatch):
    """The stream lookup of every call takes torch's public way where its private short cut is gone."""
    class Stream:
        cuda_stream = 0x5170
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        with monkeypatch.context() as m:
            m.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
            m.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0xBAD, raising=False)
            assert P._stream(None) == 0xBAD
            m.delattr(torch._C, name)
            assert P._stream(None) == 0x5170
