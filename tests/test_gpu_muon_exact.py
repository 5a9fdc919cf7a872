"""moe_expert_update_muon: X itself against 64 bits, at most three times as far from it as a model of the library's roundings is.

Where parameters are zero, the learning rate and the scale one and there is no decay, fp32 parameters (or the fp32 master copy) end as
-X. The model (muon_model) rounds what the library says it rounds, so the two are about as far from the definition; three times
leaves room for other orders of the sums. For these matrices that is some 4e-3 in fp16 and 6e-6 in two parts, 50 times less than a
coefficient 1% off and a hundred times less than a missing step change X."""
import pytest
import torch

from muon_model import apart, definition, rounded
from paper_2506_02965_amd import pcmoe as P

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)


def update(d, f, G, dtype, precise, master, steps=5, coef=COEF, nesterov=True, momentum=0.95, spike=0.0, seed=0):
    """[(X, u, sides)] of all matrices after an update, u in 64 bits from the momentum that the library left."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + d + 31 * f)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    sides = ((f, d), (f, d), (d, f))

    def normal(*s, std):
        return torch.randn(*s, device="cuda", generator=gen) * std

    def gradient(a, b):
        return (normal(G, a, b, std=1e-3) + spike * normal(G, a, 4, std=1e-3) @ normal(G, 4, b, std=1.0).contiguous()).to(dt)
    w = [torch.zeros(G, a, b, dtype=dt, device="cuda") for a, b in sides]
    g = [gradient(a, b) for a, b in sides]
    m = normal(3 * G * f * d, std=2e-3)
    mp = torch.zeros_like(m) if master else None
    opt = P.make_muon(lr=1.0, momentum=momentum, weight_decay=0.0, scale=1.0, nesterov=nesterov, steps=steps, coefficients=coef,
                      precise=precise)
    desc = P.make_desc(1, d, f, G, 1, dtype=dtype)
    ws = torch.empty(P.moe_workspace_size(desc, P.MOE_WS_UPDATE_MUON_PRECISE if precise else P.MOE_WS_UPDATE_MUON),
                     dtype=torch.uint8, device="cuda")
    P.moe_expert_update_muon(desc, opt, *w, *g, mp, m, ws, ws.numel())
    n, out = d * f, []
    for t in range(3):
        for i in range(G):
            at = (t * G + i) * n
            x = -(mp[at:at + n].view(sides[t]) if master else w[t][i])
            if master:
                assert torch.equal(w[t][i], (-x).to(dt))
            u = m[at:at + n].view(sides[t]).double()
            out.append((x, g[t][i].double() + float(opt.momentum) * u if nesterov else u))
    return out, opt


def check(d, f, G, dtype="f32", precise=False, master=None, picks=None, **kw):
    master = dtype == "bf16" if master is None else master
    out, opt = update(d, f, G, dtype, precise, master, **kw)
    coef = (float(opt.a), float(opt.b), float(opt.c))
    for k, (x, u) in enumerate(out):
        if picks is not None and k not in picks:
            continue
        want = definition(u, float(opt.eps), opt.steps, coef)
        model = apart(rounded(u, float(opt.eps), opt.steps, coef, precise), want)
        off = apart(x, want)
        assert off <= 3 * model + 2.0 ** -23, (k, off, model)


SIZES = [(128, 128, 1), (128, 384, 2), (384, 128, 1), (256, 640, 3), (640, 256, 1), (512, 512, 2), (1024, 384, 1), (1408, 256, 1),
         (384, 512, 2), (512, 640, 2)]


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,f,G", SIZES)
def test_sizes(d, f, G, dtype, precise):
    check(d, f, G, dtype, precise)


@pytest.mark.parametrize("opt", [dict(steps=1), dict(steps=2), dict(steps=3), dict(steps=4), dict(steps=6), dict(steps=9),
                                 dict(nesterov=False), dict(momentum=0.0), dict(coef=(1.5, -0.5, 0.0)), dict(coef=(2.0, -1.5, 0.5)),
                                 dict(coef=(1.0, 0.0, 0.0)), dict(spike=0.5), dict(spike=3.0)], ids=str)
@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("d,f", [(256, 384), (384, 384)])
def test_settings(opt, precise, d, f):
    check(d, f, 2, "f32", precise, **opt)


@pytest.mark.parametrize("d,f,G,dtype,precise", [
    (1024, 1536, 9, "bf16", False), (1536, 1024, 9, "f32", True), (640, 896, 16, "bf16", True), (896, 640, 16, "f32", False),
    (1024, 1280, 2, "bf16", False), (640, 2176, 1, "f32", True), (256, 256, 24, "bf16", False), (2304, 2560, 1, "bf16", False)])
def test_tiles_of_every_size(d, f, G, dtype, precise):
    check(d, f, G, dtype, precise, picks=(0, G - 1, G, 2 * G + G // 2, 3 * G - 1))


@pytest.mark.parametrize("d,f,G,dtype,precise", [(128, 2048, 1, "f32", True), (4096, 128, 2, "bf16", False),
                                                 (256, 3200, 2, "bf16", True), (2176, 384, 1, "bf16", False),
                                                 (128, 1152, 8, "f32", False), (128, 11264, 8, "bf16", False)])
def test_long_rows_split_their_sums(d, f, G, dtype, precise):
    check(d, f, G, dtype, precise, picks=(0, 3 * G - 1))


def test_several_passes():
    check(128, 256, 256, "bf16", picks=(0, 200, 600, 767))
    check(256, 640, 256, "f32", picks=(0, 500, 767))
