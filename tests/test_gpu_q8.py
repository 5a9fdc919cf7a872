"""8-bit rows and the experts in 8-bit integers against 64 bits.

Tolerances: half a step of bf16 (eps / 2 of the value) on an output, 16 fp32 roundings (2^-24) of the
magnitudes that go into it, and, where an H lies so near the border between two codes that 64 fp32 roundings of it decide,
the change of an output by one step of that code."""
import pytest
import torch

from paper_2506_02965_amd import pcmoe as P

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


def pack(w, dtype):
    n, rows, cols = w.shape
    codes = torch.full((n, rows, cols), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((n, rows), 9.0, device="cuda")
    P.moe_q8_pack(n, rows, cols, dtype, w, codes, scales)
    return codes, scales


def codes_of(v):
    """Codes and largest magnitudes of 64-bit rows. 127 |v| and its remainder are exact for fp32 and bf16 values."""
    m = v.abs().amax(-1, keepdim=True)
    a = 127 * v.abs()
    low = torch.floor(a / torch.where(m > 0, m, torch.ones_like(m)))
    twice = 2 * (a - low * m)
    code = low + ((twice > m) | ((twice == m) & (low % 2 == 1)))
    return torch.copysign(code, v) * (m > 0), m[..., 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,rows,cols", [(1, 1, 128), (3, 7, 256), (2, 130, 1408), (1, 33, 4096), (1, 5, 14336), (2, 3, 32256)])
def test_pack_and_unpack(n, rows, cols, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(n * rows + cols)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    w = torch.randn(n, rows, cols, device="cuda", generator=g).to(dt)
    w[0, 0, 1:5] = torch.tensor([0.5, -0.5, 0.25, -1.0], device="cuda").to(dt) * w[0, 0].abs().max()   # ties
    codes, scales = pack(w, dtype)
    want, m = codes_of(w.double())
    assert torch.equal(codes.double(), want)
    assert torch.equal(scales, (m / 127).float())
    back = torch.full_like(w, 5.0)
    P.moe_q8_unpack(n, rows, cols, dtype, codes, scales, back)
    assert torch.equal(back, (codes.float() * scales[..., None]).to(dt))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_out_of_the_ordinary(dtype):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    w = torch.randn(1, 12, 384, device="cuda").to(dt)
    w[0, 0] = 0.0
    w[0, 1] = -0.0
    w[0, 2] *= 1e38 / w[0, 2].abs().max()
    w[0, 3] *= 1e-38
    w[0, 4, 7] = float("nan")
    w[0, 5, 8] = float("inf")
    w[0, 6, 300] = -float("inf")
    w[0, 7] = (torch.randint(-254, 255, (384,), device="cuda") * 0.5).to(dt)       # every code and every tie
    w[0, 7, 0] = 127.0
    w[0, 8] = torch.zeros(384)
    w[0, 8, 383] = -3.0
    w[0, 9] = 2.0 ** -130 if dtype == "f32" else 2.0 ** -126
    codes, scales = pack(w, dtype)
    fine = [0, 1, 2, 3, 7, 8, 9, 10, 11]
    want, m = codes_of(w.double())
    assert torch.equal(codes[0, fine].double(), want[0, fine])
    s = (m / 127).float()
    assert ((scales[0, fine] - s[0, fine]).abs() <= 2.0 ** -149).all()        # equal, or one step of a subnormal number
    assert torch.isnan(scales[0, [4, 5, 6]]).all() and not codes[0, [4, 5, 6]].any()


class Experts:
    def __init__(self, T, d, f, E, k=1, shared=0, local=None, begin=0, counts=None, seed=0, x_scale=1.0):
        self.T, self.d, self.f, self.k, self.S = T, d, f, k, shared
        self.E = E if local is None else local
        self.G = self.E + shared
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + T + 7 * d + 13 * f + E)

        def normal(*s, std=1.0):
            return (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()
        self.gate = pack(normal(self.G, f, d, std=d ** -0.5), "bf16")
        self.up = pack(normal(self.G, f, d, std=d ** -0.5), "bf16")
        self.down = pack(normal(self.G, d, f, std=f ** -0.5), "bf16")
        self.x, self.x_perm = normal(T, d, std=x_scale), normal(T * k, d, std=x_scale)
        if counts is None:
            idx = torch.rand(T, E, device="cuda", generator=g).topk(k, 1).indices
            counts = torch.bincount(idx.reshape(-1), minlength=E)[begin:begin + self.E].tolist()
        assert len(counts) == self.E and sum(counts) <= T * k and max(counts) <= T
        self.offsets = torch.zeros(self.E + 1, dtype=torch.int32, device="cuda")
        self.offsets[1:] = torch.tensor(counts, device="cuda").cumsum(0)
        self.off = [0]
        for n in counts:
            self.off.append(self.off[-1] + n)
        self.desc = P.make_desc(T, d, f, E, k, begin, local, shared)
        self.ws = torch.full((P.moe_workspace_size(self.desc, P.MOE_WS_FFN_Q8),), 0x7f, dtype=torch.uint8, device="cuda")

    def run(self, y=None):
        y = torch.full((self.T * (self.k + self.S), self.d), 3.0, dtype=torch.bfloat16, device="cuda") if y is None else y
        P.moe_expert_ffn_q8(self.desc, self.x, self.x_perm, self.offsets, *self.gate, *self.up, *self.down, y, self.ws,
                            self.ws.numel())
        return y

    def groups(self):
        for g in range(self.E):
            if self.off[g + 1] > self.off[g]:
                yield g, slice(self.off[g], self.off[g + 1]), self.x_perm[self.off[g]:self.off[g + 1]]
        for s in range(self.S):
            yield self.E + s, slice(self.T * (self.k + s), self.T * (self.k + s + 1)), self.x

    def check(self):
        y = self.run()
        for g, rows, x in self.groups():
            xc, xm = codes_of(x.double())

            def times(c, scale, w):
                return (c @ w[0][g].double().t()) * (scale[:, None].double() * w[1][g].double())
            xs = (xm / 127).float()
            a, u = times(xc, xs, self.gate), times(xc, xs, self.up)
            h = a / (1 + torch.exp(-a)) * u
            hc, hm = codes_of(h)
            q = 127 * h / hm.clamp(min=1e-300)[:, None]
            near = ((q.abs() - torch.floor(q.abs()) - 0.5).abs() <= 64 * U32 * q.abs().clamp(min=1.0)).double()
            ref = times(hc, hm / 127, self.down)
            mag = (hc.abs() @ self.down[0][g].double().abs().t()) * (hm[:, None] / 127 * self.down[1][g].double())
            step = (near @ self.down[0][g].double().abs().t()) * (hm[:, None] / 127 * self.down[1][g].double())
            got = y[rows].double()
            tol = torch.finfo(torch.bfloat16).eps / 2 * ref.abs() + 16 * U32 * (ref.abs() + mag) + 1.01 * step
            # the row's scale hangs on its largest H, 64 fp32 roundings off at most
            tol = tol + 64 * U32 * ref.abs()
            assert ((got - ref).abs() <= tol).all(), (g, float(((got - ref).abs() / tol).max()))
        n = self.off[-1]
        assert (y[n:self.T * self.k] == 3.0).all()        # rows that no hosted expert owns
        return y


@pytest.mark.parametrize("T,d,f,E,k,shared", [
    (1, 128, 128, 1, 1, 0), (1, 256, 384, 8, 2, 1), (2, 640, 128, 4, 4, 0), (5, 128, 1408, 4, 1, 2), (16, 384, 256, 2, 2, 0),
    (17, 256, 256, 3, 2, 1), (40, 1408, 384, 64, 6, 2), (64, 512, 640, 4, 2, 0), (65, 256, 896, 1, 1, 1),
    (127, 384, 512, 3, 1, 0), (129, 512, 384, 2, 1, 1), (300, 256, 640, 8, 8, 0), (600, 384, 256, 4, 2, 1),
    (1100, 256, 1024, 2, 1, 0), (1537, 896, 384, 5, 2, 1)])
def test_experts(T, d, f, E, k, shared):
    Experts(T, d, f, E, k, shared).check()


@pytest.mark.parametrize("T,counts", [(40, [0, 40, 0, 1]), (40, [0, 0, 0, 0]), (300, [0, 300, 16, 0, 1, 255, 0]),
                                      (513, [513, 0, 0, 512]), (700, [1] * 16), (2100, [2049, 3, 0, 128, 256])])
def test_ragged_groups(T, counts):
    Experts(T, 256, 384, len(counts), 2, shared=1, counts=counts).check()


def test_shards_and_large_groups():
    Experts(90, 256, 384, 16, 4, shared=1, local=4, begin=8).check()
    Experts(3000, 512, 768, 2, 1).check()
    Experts(24, 2048, 1408, 8, 2).check()
    Experts(700, 1024, 2816, 4, 2, shared=1).check()


def test_long_rows():
    """Rows of x and of H that a workgroup codes, with and without chunks beyond those it keeps."""
    Experts(33, 2304, 1152, 2, 1).check()
    Experts(9, 4224, 4352, 2, 1, shared=1).check()
    Experts(3, 256, 20480, 1, 1).check()


@pytest.mark.parametrize("T,d,f,counts", [(1100, 4096, 4096, [1030, 70]), (1100, 4096, 4096, [512, 0]), (4160, 2176, 2048, [4100, 60]),
                                          (4160, 2176, 2048, [0, 4160])])
def test_large_tiles(T, d, f, counts):
    """Groups that the walking 256-row tiles are chosen for, in gate and up or in the down projection, whole tiles and tails."""
    Experts(T, d, f, 2, 1, counts=counts).check()


def test_many_groups():
    Experts(64, 128, 128, 256, 8, shared=3).check()


def test_rows_do_not_depend_on_each_other():
    """A row's outputs in a large call are those of a call of its own, whatever kernels run them."""
    e = Experts(400, 384, 640, 2, 1, counts=[300, 100])
    y = e.run()
    for T in (1, 9, 33, 100):
        s = Experts(T, 384, 640, 2, 1, counts=[T, 0])
        s.gate, s.up, s.down = e.gate, e.up, e.down
        s.x_perm = e.x_perm[:T].clone()
        assert torch.equal(s.run()[:T], y[:T]), T


def test_more_rows_than_a_launch_has_workgroups():
    """4.3 million rows of H: more than a launch of 2^20 workgroups takes at once."""
    T, k = 720000, 6
    e = Experts(T, 128, 128, k, k, counts=[T] * k)
    y = e.run()
    last = k * T - 50
    s = Experts(50, 128, 128, k, 1, counts=[0] * (k - 1) + [50])
    s.gate, s.up, s.down = e.gate, e.up, e.down
    s.x_perm = e.x_perm[last:].clone()
    assert torch.equal(s.run(), y[last:])


def test_broken_rows_and_weights():
    e = Experts(150, 256, 384, 2, 1, counts=[100, 50])
    clean = e.run().clone()
    e.x_perm[3, 5], e.x_perm[120, 0] = float("nan"), float("inf")
    e.x_perm[7] = 0.0
    y = e.run()
    same = [r for r in range(150) if r not in (3, 120, 7)]
    assert torch.isnan(y[[3, 120]]).all() and torch.equal(y[same], clean[same]) and not y[7].any()
    e.down[1][0, 9] = float("nan")              # a broken output channel of one expert
    y = e.run()
    assert torch.isnan(y[:100, 9]).all()
    ok = [c for c in range(256) if c != 9]
    rows = [r for r in same if r < 100]
    assert torch.equal(y[rows][:, ok], clean[rows][:, ok])
    assert torch.equal(y[[r for r in same if r >= 100]], clean[[r for r in same if r >= 100]])


def test_streams_graphs_and_guards():
    e = Experts(70, 384, 256, 4, 2, shared=1)
    y = e.run()
    n = e.ws.numel()
    whole = torch.full((n + 4096,), 0x55, dtype=torch.uint8, device="cuda")
    e.ws = whole[:n]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2 = e.run()
    s.synchronize()
    assert torch.equal(y, y2) and (whole[n:] == 0x55).all()
    out = torch.full_like(y, 3.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        e.run(out)
    for _ in range(3):
        e.x_perm.copy_(torch.randn_like(e.x_perm, dtype=torch.float32))
        e.x.copy_(torch.randn_like(e.x, dtype=torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, e.run())
