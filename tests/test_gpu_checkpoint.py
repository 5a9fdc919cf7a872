"""8-bit checkpoints of the saved activations: restored values and the tile plan, bit for bit, and a whole training step
through them."""
import math

import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import MoELayer, upload
from paper_2506_02965_amd.synth import LayerConfig, make_inputs
from gpu_util import log

pytestmark = pytest.mark.gpu


def views(saved, R, f, dt):
    es = 2 if dt == torch.bfloat16 else 4
    at = (R * 2 * f * es + 255) // 256 * 256
    return saved[:R * 2 * f * es].view(dt).view(R, 2 * f), saved[at:at + R * f * es].view(dt).view(R, f)


def quantised(v):
    """The restored values of v [R, C] in fp64, by the definition."""
    b = v.double().view(v.shape[0], -1, 32)
    fin = torch.isfinite(b)
    top = torch.where(fin, b.abs(), 0).amax(2, keepdim=True)
    m, e = torch.frexp(top)                              # 127 = 0.9921875 * 2^7
    e = torch.where(top > 0, e - 7 + (m > 0.9921875).int(), torch.full_like(e, -126)).clamp(-126, 121)
    step = torch.ldexp(torch.ones_like(top), e)
    return torch.where(fin, (b / step).round().clamp(-127, 127) * step, math.nan).view(v.shape)


CASES = [  # T, f, E, k, hosted, shared, dtype
    (1, 128, 2, 1, 2, 0, "bf16"), (1, 1408, 64, 6, 64, 2, "bf16"), (37, 384, 8, 2, 8, 1, "bf16"),
    (300, 128, 8, 2, 3, 0, "bf16"), (129, 256, 16, 4, 16, 0, "f32"), (65, 640, 8, 2, 2, 2, "f32"), (5, 128, 4, 1, 1, 1, "f32"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "T{}_f{}_E{}_k{}_host{}_S{}_{}".format(*c))
def test_restored_values(case):
    T, f, E, k, loc, S, dtype = case
    log(f"[ckpt] {case}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    R = T * (k + S)
    desc = P.make_desc(T, 128, f, E, k, 0, loc, S, dtype=dtype)
    n_loc = min(T * k, T * k * loc // E + 1) if loc < E else T * k
    gen = torch.Generator().manual_seed(T)
    offsets = torch.sort(torch.randint(0, n_loc + 1, (loc + 1,), generator=gen)).values.int()
    offsets[0], offsets[-1] = 0, n_loc
    v = (torch.randn(R, 2 * f, generator=gen) * torch.exp2(torch.randint(-40, 40, (R, 2 * f // 32), generator=gen).double())
         .repeat_interleave(32, 1)).to(dt)
    lo = torch.finfo(dt)
    v[0, :32] = 0.0
    v[0, 32:64] = -0.0
    v[-1, 0:32] = lo.max
    v[-1, 32:64] = lo.min
    v[-1, 64:96] = lo.tiny
    v[-1, 96:128] = lo.smallest_normal / 8 if dtype == "f32" else lo.tiny
    v[-1, f + 3], v[-1, f + 5], v[-1, f + 70] = math.inf, -math.inf, math.nan
    v[-1, f + 32:f + 64] = 127 * 2.0 ** -9                        # codes of exactly 127
    v[-1, f + 96:f + 128] = 127.5 * 2.0 ** -9                     # ... and just past: the next power of two
    size = P.moe_workspace_size(desc, P.MOE_WS_FFN_SAVED)
    saved = torch.randint(0, 256, (size,), generator=gen, dtype=torch.uint8).cuda()
    views(saved, R, f, dt)[0].copy_(v)
    ckpt = torch.full((P.moe_workspace_size(desc, P.MOE_WS_FFN_CKPT),), 0xA5, dtype=torch.uint8, device="cuda")
    back = torch.full((size,), 0x11, dtype=torch.uint8, device="cuda")
    P.moe_ffn_checkpoint(desc, offsets.cuda(), saved, ckpt, ckpt.numel())
    P.moe_ffn_restore(desc, offsets.cuda(), ckpt, ckpt.numel(), back)
    torch.cuda.synchronize()
    gu, h = (t.cpu() for t in views(back, R, f, dt))
    row = torch.arange(R)
    valid = (row < n_loc) | (row >= T * k)
    ref = quantised(v)
    same = (gu.double() == ref) | (torch.isnan(gu.double()) & torch.isnan(ref))
    assert bool(same[valid].all()), "restored G|U differ"
    assert bool((gu[~valid].view(torch.int16 if dtype == "bf16" else torch.int32) ==
                 (0x1111 if dtype == "bf16" else 0x11111111)).all()), "rows of no hosted expert were written"
    g, u = ref.chunk(2, 1)
    hr = torch.where(g > -700, g / (1 + torch.exp(-g)), 0.0 * g) * u
    # one rounding to the type (2^-8, 2^-24 relative, or the smallest numbers), and fp32 arithmetic of a few operations,
    # the reciprocal and exponential of the bf16 form among them, 2^-20
    fin = torch.isfinite(hr) & (hr.abs() < lo.max) & valid[:, None]
    rel = 2.0 ** -8 + 2.0 ** -20 if dtype == "bf16" else 2.0 ** -20
    floor = 1e-37 * (1 + u.abs())        # where silu(G) itself is below fp32's normal numbers
    assert bool(((h.double() - hr).abs() <= rel * hr.abs() + floor)[fin & (g > -80)].all())
    plan = views(saved, R, f, dt)[1].numel() * (2 if dtype == "bf16" else 4)
    at = (R * 2 * f * (2 if dtype == "bf16" else 4) + 255) // 256 * 256
    at += (plan + 255) // 256 * 256
    assert torch.equal(back[at:], saved[at:]), "the tile plan differs"


LAYERS = [
    LayerConfig("c1", T=300, d=256, f=384, E=8, k=2, n_shared=1, seed=7),
    LayerConfig("c2", T=1000, d=256, f=256, E=16, k=4, local_begin=4, local_count=4, router_backward=False, seed=8),
    LayerConfig("c3", T=200, d=128, f=256, E=4, k=2, dtype="f32", seed=9),
    LayerConfig("c4", T=1, d=128, f=128, E=4, k=1, seed=10),
]


@pytest.mark.parametrize("cfg", LAYERS, ids=lambda c: c.name)
def test_backward_from_a_checkpoint(cfg):
    """The backward from a checkpoint gives bit for bit what it gives from saved activations in whose place the definition's
    values were put, and gradients within 3% of the full ones: a value is kept to within 2^-8 of its block's largest, about
    0.5% of the values' norm, and dG has three such factors."""
    inp = make_inputs(cfg, with_dy=True)
    w = upload(inp)
    R, f, dt = cfg.T * (cfg.k + cfg.n_shared), cfg.f, torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
    full = MoELayer(cfg)
    full.forward(w)
    full.backward(w)
    torch.cuda.synchronize()
    shared = torch.empty_like(full.saved)
    layer = MoELayer(cfg, checkpoint=True, saved=shared)
    layer.forward(w)
    assert torch.equal(layer.y, full.y)
    gu, _ = views(layer.saved, R, f, dt)
    n = int(layer.offsets[-1])
    row = torch.arange(R)
    valid = (row < n) | (row >= cfg.T * cfg.k)
    ref = quantised(gu.cpu()[valid])
    shared.fill_(0x7f)                 # another layer's forward has used the buffer since
    layer.backward(w)
    torch.cuda.synchronize()
    back = [t.clone() for t in (layer.dx, layer.dw_gate, layer.dw_up, layer.dw_down)]
    gr, hr = views(layer.saved, R, f, dt)
    assert torch.equal(gr.cpu()[valid].double(), ref)
    h_saved = hr.clone()
    gu2, h2 = views(full.saved, R, f, dt)
    gu2[valid.cuda()] = ref.to(dt).cuda()
    h2[valid.cuda()] = h_saved[valid.cuda()]
    want = [t.clone() for t in (full.dx, full.dw_gate, full.dw_up, full.dw_down)]
    full.backward(w)
    torch.cuda.synchronize()
    for a, b, c in zip(back, (full.dx, full.dw_gate, full.dw_up, full.dw_down), want):
        assert torch.equal(a, b)
        assert float((a.float() - c.float()).norm() / c.float().norm()) <= 0.03


def test_shared_buffer_needs_checkpoint():
    cfg = LAYERS[3]
    with pytest.raises(ValueError):
        MoELayer(cfg, saved=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
