"""moe_residual_norm and its adjoint against 64 bits where the other tests' tolerances grow: rows whose mean is far above their
deviation, rows next to the end of fp32's range, and the normed output by the deviation itself.

Tolerances, elementwise, from what the kernels round (u = 2^-24, a step's half of fp32; the output's own half step is added):
- The inputs are exact. A mean is an fp64 sum of d terms here and there, at most 2 d 2^-53 of the terms' size apart, and is held in
  two fp32 parts, 2^-48 of it off: S = (2^-48 + 2 d 2^-53) mean|v| / deviation of vhat. v - mean is further off by two roundings
  relative to itself and the normalised vhat by u times: 2 (difference), 1 (1 / deviation), 1 (product), and 4 of the sum of squares, whose terms are
  squares of such differences: 8 u |vhat|. Below the normal numbers 1 / deviation is a multiple of 2^-149, two roundings more for
  deviations up to 2e38: 10. The weight's product: 11. In what follows H = 11 u.
- r = alpha x + gate post(y): 14 u of the terms' magnitudes. h adds to H |h| what r's error does, divided by the deviation: its
  own, its mean's and, times |h|, that of the deviation.
- a = dh w_pre is rounded once; mean(a) and mean(a rhat) are fp64 sums of such products (1 + 10 roundings of the mean of their
  magnitudes) and are rounded twice more; the differences, products and dr add 4. So g is off by 16 u of |dr| + rstd (|a| + mean|a| +
  |rhat| mean|a rhat|). dy likewise from b = g gate w_post, with g's bound in place of a rounding.
- Sums over tokens: fp32, the terms' own bounds and one rounding for each of T rows, 512 workgroups / 16 shares and 16 shares."""
import pytest
import torch

from paper_2506_02965_amd import pcmoe as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
H = 11


def tiny(dt):
    """Half the smallest step of the type, and of the fp32 intermediates below the normal numbers."""
    return {torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}[dt] + 8 * 2.0 ** -149


class Case:
    """Tensors of one call. gate: rows of the gate, 0 for none."""

    def __init__(self, x, y, dr, dh, pre, post, gate=0, alpha=0.75, eps=1e-5, weights=True):
        T, d = (dh if dh is not None else dr).shape
        self.T, self.d, self.dt, self.pre, self.post, self.gate = T, d, (dh if dh is not None else dr).dtype, pre, post, gate
        g = torch.Generator(device="cuda")
        g.manual_seed(T * 31 + d)

        def normal(*s, std):
            return (torch.randn(*s, device="cuda", generator=g) * std + 1.0).to(self.dt)
        self.x, self.y, self.dr, self.dh = x, y, dr, dh
        self.w_pre = normal(d, std=0.2) if weights and pre != "none" else None
        self.w_post = normal(d, std=0.2) if weights and post != "none" else None
        self.g = normal(gate, d, std=0.5) if gate else None
        self.desc = P.make_desc(T, d, 128, 1, 1, dtype="bf16" if self.dt == torch.bfloat16 else "f32")
        self.norm = P.make_norm(pre, post, eps, alpha if y is not None else 1.0, max(gate, 1))
        self.eps, self.alpha = float(self.norm.eps), float(self.norm.residual_scale)

    def new(self, *s, dtype=None):
        return torch.full(s, 7.0, device="cuda", dtype=dtype or self.dt)

    def gates(self):
        one = torch.ones(1, 1, dtype=torch.float64, device="cuda")
        return one if self.g is None else self.g.double().repeat_interleave(self.T // self.gate, 0)

    def hat(self, v, kind):
        """Normalised v and 1 / deviation, in 64 bits."""
        v = v.double()
        m = v.mean(1, keepdim=True) if kind == "layer" else 0.0
        rstd = ((v - m).square().mean(1, keepdim=True) + self.eps).rsqrt()
        return (v - m) * rstd, rstd

    def shift(self, v, kind):
        """S of the docstring."""
        if kind != "layer":
            return 0.0
        return (2.0 ** -48 + 2 * self.d * 2.0 ** -53) * v.double().abs().mean(1, keepdim=True) * self.hat(v, kind)[1]

    def weight(self, w):
        return torch.ones(self.d, dtype=torch.float64, device="cuda") if w is None else w.double()

    def check(self, name, got, ref, tol):
        err = (got.double() - ref).abs()
        tol = tol + ref.abs() * torch.finfo(got.dtype).eps / 2 + tiny(got.dtype)
        bad = ~(err <= tol)
        assert not bad.any(), (name, int(bad.sum()), float((err / tol)[bad].max()), torch.nonzero(bad)[0].tolist())

    def forward(self):
        r = self.new(self.T, self.d) if self.y is not None else None
        h = self.new(self.T, self.d) if self.pre != "none" else None
        P.moe_residual_norm(self.desc, self.norm, self.x, self.y, self.w_post, self.g, self.w_pre, r, h)
        ref, e = self.x.double(), torch.zeros_like(self.x, dtype=torch.float64)    # r and its error
        if self.y is not None:
            n, mag = self.y.double(), self.y.double().abs()
            if self.post != "none":
                n = self.hat(self.y, self.post)[0] * self.weight(self.w_post)
                mag = n.abs() + self.shift(self.y, self.post) / (14 * U) * self.weight(self.w_post).abs()
            ref, e = self.alpha * ref + self.gates() * n, 14 * U * (abs(self.alpha) * ref.abs() + self.gates().abs() * mag)
            self.check("r", r, ref, e)
        if h is not None:
            n, rstd = self.hat(ref, self.pre)
            w = self.weight(self.w_pre).abs()
            off = rstd * (e + e.mean(1, keepdim=True) + n.abs() * e.square().mean(1, keepdim=True).sqrt())
            self.check("h", h, n * self.weight(self.w_pre), w * (off + self.shift(ref, self.pre)) + H * U * w * n.abs())
        return r if r is not None else self.x, h

    def backward(self, r):
        fp32 = dict(dtype=torch.float32)
        o = dict(dx=self.new(self.T, self.d), dy=self.new(self.T, self.d) if self.y is not None else None,
                 dw_post=self.new(self.d, **fp32) if self.w_post is not None else None,
                 dgate=self.new(self.gate, self.d, **fp32) if self.gate else None,
                 dw_pre=self.new(self.d, **fp32) if self.w_pre is not None else None)
        n = P.moe_workspace_size(self.desc, P.MOE_WS_NORM_BWD)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        P.moe_residual_norm_bwd(self.desc, self.norm, self.dr, self.dh, self.y, r, self.w_post, self.g, self.w_pre, o["dx"],
                                o["dy"], o["dw_post"], o["dgate"], o["dw_pre"], ws, n)
        return o

    def adjoint(self, v, kind, w, d, e):
        """Gradient of N(v) w to v from d, whose error is e; its error; the normalised v."""
        hat, rstd = self.hat(v, kind)
        a, ea = d * w, w.abs() * (e + U * d.abs())
        mean = lambda t: t.mean(1, keepdim=True)
        ma, c = (mean(a) if kind == "layer" else 0.0), mean(a * hat)
        out = rstd * (a - ma - hat * c)
        mag = a.abs() + (mean(a.abs()) if kind == "layer" else 0.0) + hat.abs() * mean((a * hat).abs())
        err = rstd * (16 * U * mag + ea + (mean(ea) if kind == "layer" else 0.0) + hat.abs() * mean(ea * hat.abs()))
        return out, err, hat

    def check_backward(self, r):
        o = self.backward(r)
        G = self.dr.double() if self.dr is not None else torch.zeros(self.T, self.d, dtype=torch.float64, device="cuda")
        e = torch.zeros_like(G)
        sums = 1 + self.T + 32 + 16
        if self.pre != "none":
            out, err, hat = self.adjoint(r, self.pre, self.weight(self.w_pre), self.dh.double(), e)
            G, e = G + out, err + U * (G.abs() + out.abs())
            if self.w_pre is not None:
                t = self.dh.double() * hat
                self.check("dw_pre", o["dw_pre"], t.sum(0), U * (H + sums) * t.abs().sum(0)
                           + (self.dh.double().abs() * self.shift(r, self.pre)).sum(0))
        self.check("dx", o["dx"], self.alpha * G, abs(self.alpha) * (e + U * G.abs()))
        if self.y is None:
            return o
        b, eb = self.gates() * G, self.gates().abs() * (e + U * G.abs())
        hat = self.y.double()
        if self.post == "none":
            dy, edy = b, eb
        else:
            dy, edy, hat = self.adjoint(self.y, self.post, self.weight(self.w_post), b, eb)
        self.check("dy", o["dy"], dy, edy)
        if self.w_post is not None:
            t = b * hat
            self.check("dw_post", o["dw_post"], t.sum(0), (eb * hat.abs()).sum(0) + U * (H + sums) * t.abs().sum(0)
                       + (b.abs() * self.shift(self.y, self.post)).sum(0))
        if self.gate:
            w = self.weight(self.w_post)
            per = lambda v: v.view(self.gate, -1, self.d).sum(1)
            t = G * hat * w
            self.check("dgate", o["dgate"], per(t), per(e * (hat * w).abs()) + U * (H + 1 + sums) * per(t.abs())
                       + per((G * w).abs() * self.shift(self.y, self.post)))
        return o


def normals(seed, dt):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s, std=1.0, mean=0.0: (torch.randn(*s, device="cuda", generator=g) * std + mean).to(dt)


SIZES = [(1, 128), (37, 1408), (130, 2048), (1030, 512), (300, 4096), (5, 12288), (3, 22912)]


@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("pre,post", [("layer", "none"), ("layer", "layer"), ("rms", "layer"), ("layer", "rms"), ("rms", "rms")])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_by_the_deviation(T, d, pre, post, dt):
    normal = normals(T + d, dt)
    c = Case(normal(T, d, std=2.0, mean=0.3), normal(T, d, mean=-0.2), normal(T, d), normal(T, d), pre, post, gate=1)
    r, _ = c.forward()
    c.check_backward(r)


@pytest.mark.parametrize("mean", [1000.3, -3e4, 1e5])
@pytest.mark.parametrize("T,d", [(3, 384), (130, 2048), (1025, 640)])
def test_a_mean_far_above_the_deviation(T, d, mean):
    """fp32 rows that hold some 2^7 to 2^14 values within a deviation. Before the first block, so that h is of exact inputs; the
    adjoint of both norms at exact r and y."""
    normal = normals(5, torch.float32)
    x = normal(T, d, mean=mean)
    c = Case(x, None, normal(T, d), normal(T, d), "layer", "none")
    c.check_backward(c.forward()[0])
    c = Case(x, normal(T, d, mean=2 * mean), normal(T, d), normal(T, d), "layer", "layer", gate=1, alpha=0.0)
    c.forward()
    c.check_backward(x)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pre,post", [("rms", "rms"), ("layer", "layer"), ("rms", "layer")])
@pytest.mark.parametrize("T,d", [(64, 4096), (7, 256), (2, 8192)])
def test_rows_next_to_the_end_of_fp32(T, d, pre, post, dt):
    """Rows of some 2e37 and up to 3e38, of which sums over a row, and of their products with gradients, pass fp32. Column sums of
    all tokens hold what such rows add."""
    normal = normals(9, dt)
    x, y = normal(T, d), normal(T, d)
    size = torch.tensor([2e37, 6e37, 1.0, 3e36], device="cuda").repeat(T // 4 + 1)[:T, None]
    big = lambda v: (v.float() * size).clamp(-3e38, 3e38).to(dt)
    c = Case(x, big(y), normal(T, d), normal(T, d), pre, post, gate=1)
    c.check_backward(c.forward()[0])                       # y of any size, r of ordinary ones
    c = Case(big(x), y, normal(T, d), normal(T, d), pre, post, gate=1, alpha=1.0)
    r, _ = c.forward()
    c.check_backward(r)                                    # the residual stream
    c = Case(big(x), None, normal(T, d), normal(T, d), pre, "none")
    c.forward()
    c.check_backward(c.x)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("post", ["rms", "layer"])
def test_large_gradients(post, dt):
    """Products of gradients and differences up to 1e38 a term, whose sums over a row pass fp32: r and y of 1e8, dh of 1e30."""
    normal = normals(13, dt)
    T, d = 33, 2048
    c = Case(normal(T, d), normal(T, d, std=1e8), normal(T, d, std=1e29), normal(T, d, std=1e30), "rms", post, gate=1)
    c.check_backward(normal(T, d, std=1e8))


LONG = [(torch.bfloat16, 8704), (torch.bfloat16, 13312), (torch.bfloat16, 18432), (torch.bfloat16, 32640), (torch.float32, 4352),
        (torch.float32, 7680), (torch.float32, 9088), (torch.float32, 14336), (torch.float32, 23040)]


@pytest.mark.parametrize("dt,d", LONG, ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("T,gate", [(520, 520), (1030, 515), (514, 2), (2, 2), (1, 1)])
def test_long_rows_and_many_gates(dt, d, T, gate):
    """More gate rows than workgroups, each with its share of w_post's gradient, and long rows of every kernel."""
    normal = normals(d + T, dt)
    c = Case(normal(T, d, std=2.0), normal(T, d, mean=-0.2), normal(T, d), normal(T, d), "layer" if T & 2 else "rms", "rms", gate=gate)
    r, _ = c.forward()
    c.check_backward(r)


@pytest.mark.parametrize("dt,d", LONG + [(torch.bfloat16, 4096), (torch.bfloat16, 7168), (torch.float32, 3200)],
                         ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("pre,post", [("rms", "layer"), ("layer", "none"), ("none", "rms")])
def test_in_place(dt, d, pre, post):
    """dx in the place of dr or dh, dy in that of y or dh: the same bits."""
    normal = normals(d, dt)
    T = 600
    c = Case(normal(T, d), normal(T, d), normal(T, d), normal(T, d) if pre != "none" else None, pre, post, gate=3)
    r, _ = c.forward()
    want = c.backward(r)
    n = P.moe_workspace_size(c.desc, P.MOE_WS_NORM_BWD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for dx_at, dy_at in (("dr", "y"), ("dh", "y"), ("dr", "dh")):
        if pre == "none" and "dh" in (dx_at, dy_at):
            continue
        t = {k: getattr(c, k).clone() if getattr(c, k) is not None else None for k in ("dr", "dh", "y")}
        o = {k: torch.full_like(v, 7.0) for k, v in want.items() if k.startswith("d") and v is not None and k not in ("dx", "dy")}
        P.moe_residual_norm_bwd(c.desc, c.norm, t["dr"], t["dh"], t["y"], r, c.w_post, c.g, c.w_pre, t[dx_at], t[dy_at],
                                o.get("dw_post"), o.get("dgate"), o.get("dw_pre"), ws, n)
        assert torch.equal(t[dx_at], want["dx"]) and torch.equal(t[dy_at], want["dy"])
        assert all(torch.equal(o[k], want[k]) for k in o)
