"""8-bit experts whose G is next to the end of fp32's range, or far below zero: silu(G) U against 64 bits.

G is one product of codes, 127 * 127 times two scales: three roundings, and U alike; silu's factor 1 / (1 + exp(-G)) is one or
vanishes; H, its scale and its code (127 exactly) give six more, and O one product: 16 of 2^-24 with bf16's half step: numbers of
[1, 2) are 2^-7 apart, so half a step is up to 2^-8 of the value."""
import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from test_gpu_q8 import pack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x,gate,up", [(1.5e19, 2e19, 1e-30), (1.6e19, 2.1e19, 1e-33), (1.0, 50.0, 2.0), (1.0, 3e4, 2.0),
                                       (1e10, 1e20, 1e-12), (1.5e19, -2e19, 1e-30), (1e10, -1e20, 1e-12), (1.0, -3e4, 2.0)])
def test_gates_of_any_size(x, gate, up):
    d, f = 128, 128
    bf = lambda v: torch.tensor(v, dtype=torch.float64).bfloat16()
    h = torch.zeros(1, d, dtype=torch.bfloat16, device="cuda")
    h[0, 3] = bf(x)
    w = [torch.zeros(1, f, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [torch.zeros(1, d, f, dtype=torch.bfloat16, device="cuda")]
    w[0][0, 5, 3], w[1][0, 5, 3], w[2][0, 7, 5] = bf(gate), bf(up), bf(1e-9)
    q = [pack(t, "bf16") for t in w]
    desc = P.make_desc(1, d, f, 1, 1)
    ws = torch.empty(P.moe_workspace_size(desc, P.MOE_WS_FFN_Q8), dtype=torch.uint8, device="cuda")
    y = torch.full((1, d), 3.0, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    P.moe_expert_ffn_q8(desc, h, h, offsets, *q[0], *q[1], *q[2], y, ws, ws.numel())
    g = float(bf(x)) * float(bf(gate))
    silu = g / (1 + float(torch.exp(-torch.tensor(g, dtype=torch.float64))))
    want = silu * float(bf(x)) * float(bf(up)) * float(bf(1e-9))
    got = y.double()
    # far below zero silu vanishes; the kernel's factor stops at 2^-126
    left = 0.0 if g > 0 else 2.0 ** -125 * abs(g * float(bf(x)) * float(bf(up)) * float(bf(1e-9)))
    assert abs(float(got[0, 7]) - want) <= (2.0 ** -8 + 16 * 2.0 ** -24) * abs(want) + left, (float(got[0, 7]), want)
    got[0, 7] = 0.0
    assert not got.any()
