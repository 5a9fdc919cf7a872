"""Experts with 4-bit weights: packing bit for bit, and the SwiGLU passes against fp64 products of the unpacked weights.

Tolerances. bf16: H is rounded to 2^-9 (half an ulp, relative), the output again; a sum over f rounded terms of independent
signs is off by about 2^-9 of its norm: 4 * 2^-9 of the tensor's norm is allowed. fp32: sums of up to some thousand fp32
products, twice in a row: 2^-19 of the norm."""
import math

import pytest
import torch

from paper_2506_02965_amd import pcmoe as P
from paper_2506_02965_amd.layer import MoELayer, Q4Experts, upload
from paper_2506_02965_amd.synth import LayerConfig, make_inputs
from gpu_util import log

pytestmark = pytest.mark.gpu
VALUES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def pack(w, group):
    n, N, K = w.shape
    codes = torch.full((n, N // 16, K // 128, 4, 16, 4, 4), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, N // 16, K // group, 16), 5.0, dtype=torch.bfloat16, device="cuda")
    P.moe_q4_pack(n, N, K, group, "bf16" if w.dtype == torch.bfloat16 else "f32", w.cuda(), codes, scales)
    return codes, scales


def unpack_ref(codes, scales, group):
    """fp64 [n, N, K] by the header's layout, element by element of the index."""
    n, nb, kb = codes.shape[:3]
    c, N, K = codes.cpu().long(), nb * 16, kb * 128
    r, k = torch.arange(N)[:, None], torch.arange(K)[None]
    byte = c[:, r // 16, k // 128, k % 32 // 8, r % 16, k % 128 // 32, k % 8 // 2]
    code = (byte >> (4 * (k % 2))) & 15
    v = VALUES[code & 7] * (1 - 2 * (code >> 3))
    return v * scales.cpu().double()[:, r // 16, k // group, r % 16]


@pytest.mark.parametrize("shape", [(1, 16, 128), (3, 48, 256), (2, 128, 640), (5, 16, 384), (2, 2048, 1024)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pack(shape, group, dtype):
    log(f"[q4] pack {shape} group={group} {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, N, K = shape
    w = torch.randn(shape, generator=torch.Generator().manual_seed(N)).to(dt)
    w[0, 0, :group] = 0
    w[0, 1, :group] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * (group // 8))    # every midpoint
    w[0, 2, :group] = -w[0, 1, :group]
    w[0, 3, 0], w[0, 4, 1], w[0, 5, 2] = math.inf, math.nan, -math.inf
    w[0, 6, :group] = torch.finfo(dt).tiny
    w[0, 7, :group] = torch.finfo(dt).max
    codes, scales = pack(w, group)
    got = unpack_ref(codes, scales, group)
    g = w.double().view(n, N, K // group, group)
    bad = ~torch.isfinite(g).all(3)
    s = (g.abs().amax(3).float() * torch.tensor(1 / 6, dtype=torch.float32)).bfloat16()   # the definition: times fp32(1/6)
    s[bad] = math.nan
    sg = scales.cpu().permute(0, 1, 3, 2).reshape(n, N, -1)
    assert torch.equal(torch.isnan(sg), bad) and torch.equal(sg[~bad], s[~bad])
    q = torch.where(s[..., None] > 0, g / s[..., None].double(), 0.0)
    step = torch.where(q.abs() < 2, 0.5, torch.where(q.abs() < 4, 1.0, 2.0))
    q = ((q / step).round() * step).clamp(-6, 6)            # nearest, ties to the even multiple: the even code
    ref = (q * s[..., None].double()).view(n, N, K)
    ok = (~bad).repeat_interleave(group, 2)
    assert torch.equal(got[ok], ref[ok])
    assert bool(torch.isnan(got[~ok]).all())
    out = torch.full(shape, 9.0, dtype=dt, device="cuda")
    P.moe_q4_unpack(n, N, K, group, dtype, codes, scales, out)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu()[ok], got[ok].to(dt)) and bool(torch.isnan(out.cpu()[~ok]).all())


def run(T, d, f, counts, k, E, S, group, dtype, seed=1, edit=None, begin=0):
    """moe_expert_ffn_q4 with the given rows per hosted expert -> (y [R, d], reference fp64, rows that are defined)."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    loc, G, R = len(counts), len(counts) + S, T * (k + S)
    gen = torch.Generator().manual_seed(seed)
    desc = P.make_desc(T, d, f, E, k, begin, loc, S, dtype=dtype)
    x, xp = torch.randn(T, d, generator=gen).to(dt), torch.randn(T * k, d, generator=gen).to(dt)
    ws = [torch.randn(G, N, K, generator=gen) * K ** -0.5 for N, K in ((f, d), (f, d), (d, f))]
    if edit:
        edit(x, xp, ws)
    q = [pack(w.to(dt), group) for w in ws]
    off = torch.zeros(loc + 1, dtype=torch.int32)
    off[1:] = torch.tensor(counts).cumsum(0)
    n = int(off[-1])
    assert n <= T * k
    y = torch.full((R, d), 77.0, dtype=dt, device="cuda")
    scratch = torch.full((P.moe_workspace_size(desc, P.MOE_WS_FFN_Q4),), 0xFF, dtype=torch.uint8, device="cuda")
    P.moe_expert_ffn_q4(desc, group, x.cuda(), xp.cuda(), off.cuda(), *q[0], *q[1], *q[2], y, scratch, scratch.numel())
    torch.cuda.synchronize()
    wq = [unpack_ref(*t, group) for t in q]
    ref = torch.full((R, d), 77.0, dtype=torch.float64)
    groups = [(g, slice(int(off[g]), int(off[g + 1])), xp[int(off[g]):int(off[g + 1])]) for g in range(loc)]
    groups += [(loc + s, slice(T * (k + s), T * (k + s + 1)), x) for s in range(S)]
    for g, rows, xr in groups:
        a = xr.double() @ wq[0][g].t()
        ref[rows] = (a / (1 + torch.exp(-a)) * (xr.double() @ wq[1][g].t())) @ wq[2][g].t()
    row = torch.arange(R)
    return y.cpu().double(), ref, (row < n) | (row >= T * k), dict(desc=desc, x=x, xp=xp, off=off, q=q)


def check(y, ref, valid, dtype):
    assert bool((y[~valid] == 77).all()), "rows of no hosted expert were written"
    err = float((y[valid] - ref[valid]).norm() / ref[valid].norm())
    assert err <= (4 * 2.0 ** -9 if dtype == "bf16" else 2.0 ** -19), err


CASES = [  # T, d, f, rows per hosted expert, k, E, shared
    (1, 128, 128, [1], 1, 1, 0), (1, 256, 384, [0, 1, 0, 1], 2, 4, 0), (1, 128, 256, [0, 0, 0], 1, 5, 2),
    (7, 384, 128, [0, 7, 3, 0, 4], 2, 5, 1), (16, 128, 256, [16, 16], 2, 2, 0), (17, 256, 128, [17, 0, 17], 2, 3, 0),
    (33, 128, 128, [33, 1, 32], 2, 3, 1), (70, 640, 256, [5, 70, 64, 1], 2, 4, 0), (130, 256, 640, [130, 127, 3], 2, 3, 0),
    (40, 128, 128, [9, 0, 12], 4, 12, 0), (5, 128, 128, [0, 0], 2, 8, 0), (300, 128, 256, [300, 150, 150], 2, 3, 1),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "T{}_d{}_f{}_{}_S{}".format(c[0], c[1], c[2], "-".join(map(str, c[3])), c[6]))
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_experts(case, group, dtype):
    T, d, f, counts, k, E, S = case
    log(f"[q4] {case} group={group} {dtype}")
    y, ref, valid, _ = run(T, d, f, counts, k, E, S, group, dtype, begin=E - len(counts))
    if bool(valid.any()):
        check(y, ref, valid, dtype)
    else:
        assert bool((y == 77).all())


KERNELS = [  # T, d, f, rows per hosted expert, k, E, shared: K past 256 in both projections
    (1, 384, 384, [1, 0, 1], 2, 3, 1),                                    # few steps, an odd number of them
    (1, 1152, 1408, [0, 1], 1, 2, 2),                                     # K split, 32 columns
    (9, 640, 1152, [9, 4, 5], 2, 3, 0),                                   # ... 16 columns of the down projection
    (9, 4096, 1024, [9, 4, 5], 2, 3, 0),                                  # K split, 64 columns
    (12, 1024, 5120, [12, 1], 2, 2, 1),                                   # ... of both projections
    (60, 384, 512, [20, 17, 33, 16, 1, 33], 2, 6, 0),                     # 32-row chunks; 16-row chunks, four steps in flight
    (100, 640, 384, [50, 49, 97, 4], 2, 4, 1),                            # ... an odd number of steps
    (800, 640, 384, [200, 129, 31, 33, 800, 0, 7, 400], 2, 8, 0),         # 32 rows x 128 columns
    (42, 384, 1024, [3, 4, 5, 2, 0, 1, 17, 3] * 6, 5, 48, 0),             # 16-row chunks of gate/up
]


@pytest.mark.parametrize("case", KERNELS, ids=lambda c: "T{}_d{}_f{}_G{}_S{}".format(c[0], c[1], c[2], len(c[3]), c[6]))
@pytest.mark.parametrize("group,dtype", [(32, "bf16"), (64, "bf16"), (128, "bf16"), (32, "f32"), (128, "f32")])
def test_each_kernel(case, group, dtype):
    T, d, f, counts, k, E, S = case
    log(f"[q4] kernels T={T} d={d} f={f} group={group} {dtype}")
    y, ref, valid, _ = run(T, d, f, counts, k, E, S, group, dtype)
    check(y, ref, valid, dtype)


@pytest.mark.parametrize("G", [65, 256])
def test_many_experts(G):
    counts = [(3 * g + g // 64) % 4 for g in range(G)]
    y, ref, valid, _ = run(sum(counts), 128, 128, counts, 1, G, 0, 32, "bf16")
    check(y, ref, valid, "bf16")


@pytest.mark.parametrize("T", [1, 24, 200])
def test_real_widths(T):
    """The widths of the workloads, a few experts of each."""
    for d, f, group in ((2048, 1408, 128), (1024, 2816, 32), (4096, 1792, 64)):
        y, ref, valid, _ = run(T, d, f, [T, 0, T], 2, 3, 0, group, "bf16")
        check(y, ref, valid, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_non_finite_rows_and_weights(dtype):
    """A NaN or an infinity in one row reaches that row alone; a weight group of NaN scale every row of its expert alone."""
    def edit(x, xp, ws):
        xp[3, 5], xp[9, 0] = math.nan, math.inf
        ws[1][2, 7, 3] = math.nan
    y, ref, valid, _ = run(20, 128, 128, [12, 4, 4], 1, 3, 0, 32, dtype, edit=edit)
    bad = torch.zeros(20, dtype=torch.bool)
    bad[3] = bad[9] = True
    bad[16:] = True
    assert bool(torch.isnan(y[bad]).any(1).all()) and not bool(torch.isfinite(y[16:]).any())
    check(y[~bad], ref[~bad], valid[~bad], dtype)


def test_equal_calls_equal_bits_and_other_streams():
    a, _, _, s = run(70, 256, 256, [70, 69, 1], 2, 3, 1, 64, "bf16")
    side = torch.cuda.Stream()
    y = torch.full((70 * 3, 256), 77.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(P.moe_workspace_size(s["desc"], P.MOE_WS_FFN_Q4), dtype=torch.uint8, device="cuda")
    args = (s["x"].cuda(), s["xp"].cuda(), s["off"].cuda())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        P.moe_expert_ffn_q4(s["desc"], 64, *args, *s["q"][0], *s["q"][1], *s["q"][2], y, ws, ws.numel())
    side.synchronize()
    assert torch.equal(y.cpu().double(), a)


def test_layer_graph_replays():
    """forward_q4 of a small batch captured into a graph: replays with other inputs, eager work between them, equal eager."""
    cfg = LayerConfig("q", T=24, d=256, f=384, E=8, k=2, n_shared=1, backward=False, seed=5)
    w = upload(make_inputs(cfg))
    q = Q4Experts.pack(w, 64)
    layer = MoELayer(cfg, gate=P.make_gate("sigmoid", 4, 2, 2))
    layer.forward_q4(w, q)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        layer.forward_q4(w, q)
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        layer.forward_q4(w, q)
    eager = MoELayer(cfg, gate=layer.gate)
    for seed in range(4):
        w.x.copy_(torch.randn(24, 256, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.y, eager.forward_q4(w, q)), seed
        torch.cuda.synchronize()
    ref = MoELayer(cfg, gate=layer.gate)
    ref.forward(w)                                     # 4-bit weights: some 10% off the full ones
    assert float((ref.y.float() - layer.y.float()).norm() / ref.y.float().norm()) <= 0.3
