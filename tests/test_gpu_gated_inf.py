"""Gated routing of scores of +inf (a sum that passes fp32's range, or a logit_bias that forces an expert): softmax takes its
limit, in which the experts of +inf share the whole weight and the others have none, and so do sigmoid scores. In fp64 a
score of 1e4 in their place gives the same: exp(-1e4) is 0 and 1 / (1 + exp(-1e4)) is 1. Tolerances as for finite scores."""
import math

import numpy as np
import pytest
import torch

from gpu_util import log
from paper_2506_02965_amd import pcmoe as P
from test_gpu_gated import check, gate_formula, route

pytestmark = pytest.mark.gpu
E, K = 24, 4


def bias_rows():
    lb = torch.zeros(5, E)
    lb[1, 7] = math.inf                                # one forced expert
    lb[2, [3, 20]] = math.inf                          # two, in different groups
    lb[3, 8:14] = math.inf                             # more than are selected
    lb[4, 2], lb[4, 5:] = math.inf, -math.inf          # one among masked ones
    return lb


@pytest.mark.parametrize("T", [5, 500, 5000])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_infinite_scores(T, score, renorm):
    gen = torch.Generator().manual_seed(T)
    lb, balance = bias_rows(), (torch.randn(E, generator=gen) * 30).round() * 0.001
    for bias in (None, balance):
        for groups, keep, top in ((1, 1, 1), (4, 2, 2), (12, 4, 1)):
            g = dict(score=score, n_groups=groups, topk_groups=keep, group_top=top, scale=1.5)
            log(f"[gated] inf T={T} {score} renormalize={renorm} bias={bias is not None} groups={groups}/{keep} top={top}")
            _, logits, idx, gw, desc, x, _ = route(T, 128, E, K, "f32", P.make_gate(**g), renorm, bias, lb)
            assert torch.equal(logits == math.inf, (lb == math.inf).repeat_interleave(T // 5, 0))
            finite = torch.where(logits == math.inf, 1e4, logits)
            check(finite, idx, gw, bias, K, g, renorm)
            if T == 5000:
                continue
            dg = torch.randn(T, K, generator=gen)
            dl, dw = torch.empty(T, E, device="cuda"), torch.empty(E, 128, device="cuda")
            ws = torch.empty(max(1, P.moe_workspace_size(desc, P.MOE_WS_ROUTE_BWD)), dtype=torch.uint8, device="cuda")
            P.moe_route_gated_bwd(desc, P.make_gate(**g), x.cuda(), logits.cuda(), idx.cuda(), gw.cuda(), dg.cuda(), dl, dw,
                                  ws, ws.numel())
            torch.cuda.synchronize()
            ref = gate_formula(finite.double(), idx.long(), dg.double(), gw.double(), score, renorm, 1.5)
            size = np.maximum((gw.double() * dg.double()).abs().amax(1, keepdim=True).numpy(), 1e-30)
            assert np.all(np.abs(dl.cpu().double().numpy() - ref.numpy()) <= 32 * 2.0 ** -24 * size)


@pytest.mark.parametrize("case", [(300, 8), (1000, 24), (2100, 64), (700, 66), (4100, 256)], ids=lambda c: "T{}_E{}".format(*c))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_gradients(case, dtype):
    """dW = dlogits^T x where some of dgate is infinite or NaN: infinities and NaN where the fp64 product has them, with the
    same signs, and the other experts' rows as without them."""
    T, n_experts = case
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(T)
    log(f"[gated grad] inf {case} {dtype}")
    gate = P.make_gate("sigmoid")
    _, logits, idx, gw, desc, x, _ = route(T, 128, n_experts, 2, dtype, gate, False)
    dg = torch.randn(T, 2, generator=gen)
    dg[5, 0], dg[T // 2, 1], dg[T - 1, 0] = math.inf, -math.inf, math.nan
    dl, dw = torch.empty(T, n_experts, device="cuda"), torch.empty(n_experts, 128, device="cuda")
    ws = torch.empty(max(1, P.moe_workspace_size(desc, P.MOE_WS_ROUTE_BWD)), dtype=torch.uint8, device="cuda")
    P.moe_route_gated_bwd(desc, gate, x.cuda(), logits.cuda(), idx.cuda(), gw.cuda(), dg.cuda(), dl, dw, ws, ws.numel())
    torch.cuda.synchronize()
    got, ref = dw.cpu().double(), dl.cpu().double().t() @ x.double()
    assert bool(torch.isinf(dl.cpu()).any()) and x.dtype == dt
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got == math.inf, ref == math.inf)
    assert torch.equal(got == -math.inf, ref == -math.inf)
    rows = torch.isfinite(ref).all(1)
    assert float((got[rows] - ref[rows]).norm() / ref[rows].norm()) <= 2e-6
