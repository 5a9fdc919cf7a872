"""training_footprint of layers updated along their orthogonalised momentum, against the buffers that the layer allocates."""
import os

import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import LayerWeights, MoELayer, training_footprint
from paper_2506_02965_amd.synth import LayerConfig

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libpcmoe.so not built")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("master", [True, False])
@pytest.mark.parametrize("precise", [True, False])
def test_state_of_the_orthogonalised_update(dtype, master, precise):
    cfg = LayerConfig("h", T=40, d=128, f=256, E=4, k=2, n_shared=1, dtype=dtype)
    layer, G = MoELayer(cfg, device="cpu"), cfg.n_groups
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    w = LayerWeights(None, None, None, 1, *(torch.zeros(G, *s, dtype=dt) for s in ((256, 128), (256, 128), (128, 256))))
    layer.init_muon_state(w, master=master, precise=precise)
    size = lambda *ts: sum(t.numel() * t.element_size() for t in ts if t is not None)
    state = size(w.w_gate, w.w_up, w.w_down, layer.dw_gate, layer.dw_up, layer.dw_down, layer.muon_m, layer.muon_master)
    plain = training_footprint(cfg, cfg.E, master=master)
    muon = training_footprint(cfg, cfg.E, master=master, update="muon_precise" if precise else "muon")
    assert muon["expert_state"] == state
    assert muon["update_ws"] == size(layer.ws_muon)
    assert muon["total"] - plain["total"] == muon["update_ws"] + state - plain["expert_state"]
    assert plain == training_footprint(cfg, cfg.E, master=master, update="adamw") and "update_ws" not in plain
    with pytest.raises(ValueError, match="update"):
        training_footprint(cfg, cfg.E, update="sgd2")
