"""moe_residual_norm and its adjoint against 64 bits.

Tolerances, elementwise: half a step of the output's type relative to the value, and COUNT roundings of fp32 (2^-24 each)
of the sum of the magnitudes that go into it. A value passes at most 12 fp32 roundings beside its sums (mean, deviation, two
products, residual); a row sum of fp32 terms adds 64 chained additions of a thread at the most and 16 across the threads, a
sum over tokens those of a workgroup's rows, of the workgroups' sums and of 16 shares."""
import pytest
import torch

from paper_2506_02965_amd import pcmoe as P

pytestmark = pytest.mark.gpu
COUNT = 96
U32 = 2.0 ** -24


def half_step(dt):
    return torch.finfo(dt).eps / 2


def close(got, ref, mag, count=COUNT):
    err = (got.double() - ref).abs()
    tol = half_step(got.dtype) * ref.abs() + count * U32 * mag
    bad = ~((err <= tol) | (got.double() == ref) | (torch.isnan(ref) & torch.isnan(got)))     # equal infinities differ by NaN
    assert not bad.any(), (int(bad.sum()), float((err / tol.clamp(min=1e-300))[bad].max()))


class Case:
    def __init__(self, T, d, pre, post, gate=0, alpha=1.0, dtype="bf16", weights=True, first=False, seed=0):
        self.T, self.d, self.pre, self.post, self.gate, self.alpha, self.first = T, d, pre, post, gate, alpha, first
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + T * 7919 + d)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32

        def normal(*s, std=1.0, mean=0.0):
            return (torch.randn(*s, device="cuda", generator=g) * std + mean).to(self.dt)
        self.x = normal(T, d, std=2.0, mean=0.3)
        self.y = None if first else normal(T, d, mean=-0.2)
        self.w_pre = normal(d, std=0.2, mean=1.0) if weights and pre != "none" else None
        self.w_post = normal(d, std=0.2, mean=1.0) if weights and post != "none" else None
        self.g = normal(gate, d, std=0.5, mean=1.0) if gate else None
        self.dr, self.dh = normal(T, d), normal(T, d) if pre != "none" else None
        self.desc = P.make_desc(T, d, 128, 1, 1, dtype=dtype)
        self.norm = P.make_norm(pre, post, 1e-5, alpha, max(gate, 1))
        self.eps = float(self.norm.eps)
        self.alpha = float(self.norm.residual_scale)

    def new(self, *s, dtype=None):
        return torch.full(s, 7.0, device="cuda", dtype=dtype or self.dt)

    def forward(self):
        r = None if self.first else self.new(self.T, self.d)
        h = self.new(self.T, self.d) if self.pre != "none" else None
        P.moe_residual_norm(self.desc, self.norm, self.x, self.y, self.w_post, self.g, self.w_pre, r, h)
        return r, h

    def backward(self, r, dr="given", **out):
        o = dict(dx=self.new(self.T, self.d), dy=None if self.first else self.new(self.T, self.d),
                 dw_post=self.new(self.d, dtype=torch.float32) if self.w_post is not None else None,
                 dgate=self.new(self.gate, self.d, dtype=torch.float32) if self.gate else None,
                 dw_pre=self.new(self.d, dtype=torch.float32) if self.w_pre is not None else None)
        o.update(out)
        n = P.moe_workspace_size(self.desc, P.MOE_WS_NORM_BWD)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        P.moe_residual_norm_bwd(self.desc, self.norm, self.dr if dr == "given" else None, self.dh, self.y, r, self.w_post,
                                self.g, self.w_pre, o["dx"], o["dy"], o["dw_post"], o["dgate"], o["dw_pre"], ws, n)
        return o

    # ---- 64 bits
    def f64(self, v, kind, w):
        """N(v), and the magnitude that its rounding errors scale with."""
        v = v.double()
        if kind == "none":
            return v, v.abs()
        mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
        rstd = ((v - mean) ** 2).mean(1, keepdim=True).add(self.eps).rsqrt()
        w = torch.ones(self.d, dtype=torch.float64, device="cuda") if w is None else w.double()
        return (v - mean) * rstd * w, (v.abs() + mean.abs()) * rstd * w.abs()

    def gates(self):
        if self.g is None:
            return torch.ones(1, 1, dtype=torch.float64, device="cuda")
        return self.g.double().repeat_interleave(self.T // self.gate, 0)

    def check_forward(self):
        r, h = self.forward()
        ref, mag = self.x.double(), self.x.double().abs()
        if not self.first:
            n, m = self.f64(self.y, self.post, self.w_post)
            ref, mag = self.alpha * ref + self.gates() * n, abs(self.alpha) * mag + self.gates().abs() * m
            close(r, ref, mag)
        if h is not None:
            n, m = self.f64(ref, self.pre, self.w_pre)
            rstd = n.abs().sum() * 0 + (m / (ref.abs() + 1e-30)).amax(1, keepdim=True)   # bounds w / deviation
            close(h, n, m + rstd * mag)
        return r if r is not None else self.x, h

    def check_backward(self, r, dr="given"):
        o = self.backward(r, dr)
        leaves = {"r": r.double().requires_grad_(True)}
        for k in ("y", "w_post", "w_pre", "g"):
            v = getattr(self, k)
            if v is not None:
                leaves[k] = v.double().requires_grad_(True)
        f = {k: leaves.get(k) for k in ("y", "w_post", "w_pre", "g")}

        def norm(v, kind, w):
            if kind == "none":
                return v
            m = v.mean(1, keepdim=True) if kind == "layer" else 0
            n = (v - m) * ((v - m) ** 2).mean(1, keepdim=True).add(self.eps).rsqrt()
            return n if w is None else n * w
        G = torch.zeros_like(leaves["r"]) if dr != "given" else self.dr.double()
        mag_g = G.abs()
        if self.pre != "none":
            # gradients through h, and the magnitudes that go into them
            h = norm(leaves["r"], self.pre, f["w_pre"])
            wanted = [leaves["r"]] + ([leaves["w_pre"]] if f["w_pre"] is not None else [])
            got = torch.autograd.grad(h, wanted, self.dh.double())
            G = G + got[0]
            with torch.no_grad():
                v = r.double()
                m = v.mean(1, keepdim=True) if self.pre == "layer" else torch.zeros_like(v[:, :1])
                rstd = ((v - m) ** 2).mean(1, keepdim=True).add(self.eps).rsqrt()
                hat = (v.abs() + m.abs()) * rstd
                a = self.dh.double().abs() * (1 if f["w_pre"] is None else self.w_pre.double().abs())
                mag_g = mag_g + rstd * (a + a.mean(1, keepdim=True) + hat * (a * hat).mean(1, keepdim=True))
                if f["w_pre"] is not None:
                    close(o["dw_pre"], got[1], (self.dh.double().abs() * hat).sum(0), self.sums())
        close(o["dx"], self.alpha * G, abs(self.alpha) * mag_g)
        if self.first:
            return o
        n = norm(leaves["y"], self.post, f["w_post"])
        b = n if f["g"] is None else n * f["g"].repeat_interleave(self.T // self.gate, 0)
        names = [k for k in ("y", "w_post", "g") if f[k] is not None]
        got = dict(zip(names, torch.autograd.grad(b, [leaves[k] for k in names], G)))
        with torch.no_grad():
            gm = mag_g * self.gates().abs()
            if self.post == "none":
                mag_y, hat = gm, self.y.double().abs()
            else:
                v = self.y.double()
                m = v.mean(1, keepdim=True) if self.post == "layer" else torch.zeros_like(v[:, :1])
                rstd = ((v - m) ** 2).mean(1, keepdim=True).add(self.eps).rsqrt()
                hat = (v.abs() + m.abs()) * rstd
                a = gm * (1 if f["w_post"] is None else self.w_post.double().abs())
                mag_y = rstd * (a + a.mean(1, keepdim=True) + hat * (a * hat).mean(1, keepdim=True))
            close(o["dy"], got["y"], mag_y, 2 * COUNT)
            if f["w_post"] is not None:
                close(o["dw_post"], got["w_post"], (gm * hat).sum(0), 2 * self.sums())
                hat = hat * self.w_post.double().abs()
            if f["g"] is not None:
                close(o["dgate"], got["g"], (mag_g * hat).view(self.gate, -1, self.d).sum(1), 2 * self.sums())
        return o

    def sums(self):
        """Roundings of a sum over tokens: COUNT of a term, its workgroup's rows (up to twice the mean where gate
        rows are shared out), the workgroups' sums and 16 shares."""
        return COUNT + 2 * self.T / max(1, min(512, self.T // 4)) + 1 + 512 / 16 + 16


SIZES = [(1, 128), (1, 4096), (2, 256), (3, 384), (5, 640), (37, 1408), (130, 2048), (513, 128), (1030, 512), (300, 4096),
         (4, 7168), (1025, 2560)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("pre,post", [("rms", "rms"), ("layer", "none"), ("rms", "layer"), ("none", "rms"),
                                      ("layer", "layer"), ("none", "none")])
def test_forward_and_backward(T, d, pre, post, dtype):
    c = Case(T, d, pre, post, gate=1, alpha=0.75, dtype=dtype)
    r, _ = c.check_forward()
    c.check_backward(r)


@pytest.mark.parametrize("T,d,gate", [(1, 256, 1), (6, 384, 6), (6, 384, 3), (6, 384, 2), (777, 128, 7), (777, 128, 777),
                                      (777, 128, 111), (2048, 128, 1024), (2048, 128, 2048), (1000, 256, 0), (600, 640, 300),
                                      (2049, 128, 3)])
@pytest.mark.parametrize("post", ["none", "rms", "layer"])
def test_gates(T, d, gate, post):
    for dtype in ("bf16", "f32"):
        c = Case(T, d, "rms", post, gate=gate, alpha=1.0, dtype=dtype, seed=3)
        r, _ = c.check_forward()
        c.check_backward(r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 128), (65, 512), (1100, 384)])
def test_before_the_first_and_after_the_last_block(T, d, dtype):
    c = Case(T, d, "rms", "none", dtype=dtype, first=True)
    r, _ = c.check_forward()
    assert r is c.x
    c.check_backward(r)
    c.check_backward(r, dr=None)
    c = Case(T, d, "layer", "rms", dtype=dtype, weights=False)     # no weights, and nothing but h uses r
    r, _ = c.check_forward()
    c.check_backward(r, dr=None)


@pytest.mark.parametrize("dtype,d", [("bf16", 16384), ("bf16", 20480), ("bf16", 32256), ("f32", 8320), ("f32", 16512),
                                     ("f32", 22912)])
def test_long_rows(dtype, d):
    """Rows that need more chunks a thread and larger workgroups, up to the longest that a descriptor takes."""
    for T in (3, 1029):
        c = Case(T, d, "rms", "layer", gate=1, dtype=dtype)
        r, _ = c.check_forward()
        c.check_backward(r)
        del c


def test_extreme_rows():
    for dtype in ("bf16", "f32"):
        for pre, post in (("rms", "rms"), ("layer", "layer")):
            c = Case(8, 256, pre, post, gate=1, dtype=dtype)
            c.x[0], c.y[0] = 0.0, 0.0                        # nothing: h is 0, not NaN
            c.y[1], c.x[1] = c.y[1] * 1e30, c.x[1] * 1e-30   # squares pass fp32
            c.y[2], c.x[2] = c.y[2] * 1e-30, c.x[2] * 1e-30  # ... and vanish in it
            c.x[3] = c.x[3] * 1e25
            c.x[4, 5] = float("nan")
            c.x[5, 7] = float("inf")
            c.y[6] = c.y[6] * 0.01 + 3.0                     # a mean far above the deviation
            r, h = c.forward()
            n, m = c.f64(c.y, post, c.w_post)
            ref = c.alpha * c.x.double() + c.gates() * n
            close(r, ref, c.x.double().abs() + c.gates().abs() * m)
            fine = [0, 1, 2, 3, 6, 7]
            n, m = c.f64(ref[fine], pre, c.w_pre)
            rstd = (m / (ref[fine].abs() + 1e-300)).nan_to_num(0.0).amax(1, keepdim=True)
            mag = (c.x.double().abs() + c.gates().abs() * c.f64(c.y, post, c.w_post)[1])[fine]
            close(h[fine], n, m + rstd * mag)
            assert torch.isnan(h[4]).all()
            assert torch.isnan(h[5, 7])
            if pre == "rms":                                 # finite numbers over an infinite deviation
                assert not h[5, :7].any() and not h[5, 8:].any()
            o = c.backward(r)
            assert torch.isfinite(o["dx"][fine]).all() and torch.isfinite(o["dy"][[0, 2, 3, 6, 7]]).all()
            assert torch.isnan(o["dx"][4]).all()


def test_difference_quotients():
    """The adjoint against central differences of the fp32 forward: sums of 384 x 24 products with a random direction."""
    c = Case(24, 384, "rms", "layer", gate=3, alpha=0.5, dtype="f32", seed=11)
    r, _ = c.forward()
    o = c.backward(r)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    for name, grad in (("x", o["dx"]), ("y", o["dy"]), ("w_post", o["dw_post"]), ("w_pre", o["dw_pre"]), ("g", o["dgate"])):
        v0 = getattr(c, name)
        t = torch.randn(v0.shape, device="cuda", generator=gen)
        step, val = 2.0 ** -6, []
        for s in (step, -step):
            setattr(c, name, v0 + s * t)
            rr, hh = c.forward()
            val.append((rr.double() * c.dr.double()).sum() + (hh.double() * c.dh.double()).sum())
        setattr(c, name, v0)
        diff = float((val[0] - val[1]) / (2 * step))
        want = float((grad.double() * t.double()).sum())
        # third derivatives of values of order one: step^2 of the terms' absolute sum; rounding: 2^-24 of it over the step
        size = float((grad.double() * t.double()).abs().sum()) + float(c.dr.double().abs().sum())
        assert abs(diff - want) <= size * (step ** 2 + COUNT * U32 / step), (name, diff, want)


def test_in_place_strides_and_streams():
    c = Case(300, 512, "rms", "rms", gate=1, dtype="bf16")
    r, h = c.forward()
    x2, y2 = c.x.clone(), c.y.clone()
    h2 = c.new(c.T, c.d)
    P.moe_residual_norm(c.desc, c.norm, x2, c.y, c.w_post, c.g, c.w_pre, x2, h2)
    assert torch.equal(x2, r) and torch.equal(h2, h)
    P.moe_residual_norm(c.desc, c.norm, c.x, y2, c.w_post, c.g, c.w_pre, y2, h2)
    assert torch.equal(y2, r)
    with pytest.raises(ValueError):
        P.moe_residual_norm(c.desc, c.norm, c.x.t().contiguous().t(), c.y, c.w_post, c.g, c.w_pre, r, h)
    o = c.backward(r)
    dr, y = c.dr.clone(), c.y.clone()
    n = P.moe_workspace_size(c.desc, P.MOE_WS_NORM_BWD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    P.moe_residual_norm_bwd(c.desc, c.norm, dr, c.dh, y, r, c.w_post, c.g, c.w_pre, dr, y, o["dw_post"], o["dgate"],
                            o["dw_pre"], ws, n)
    assert torch.equal(dr, o["dx"]) and torch.equal(y, o["dy"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        h3, r3 = torch.empty_like(h), torch.empty_like(r)
        P.moe_residual_norm(c.desc, c.norm, c.x, c.y, c.w_post, c.g, c.w_pre, r3, h3)
    s.synchronize()
    assert torch.equal(h3, h) and torch.equal(r3, r)


@pytest.mark.parametrize("pre", ["none", "layer"])
def test_backward_without_y(pre):
    """Neither a post norm nor a gate reads y: dy is written without it, and r only where a pre norm reads it."""
    c = Case(70, 384, pre, "none", alpha=0.5, dtype="bf16")
    r, _ = c.forward()
    o = c.backward(r)
    c.y = None
    other = c.backward(r if pre != "none" else None)
    assert torch.equal(o["dx"], other["dx"]) and torch.equal(o["dy"], other["dy"])
    assert not (o["dy"] == 7.0).all()


def test_graph_replays():
    c = Case(130, 640, "layer", "rms", gate=2, dtype="bf16")
    n = P.moe_workspace_size(c.desc, P.MOE_WS_NORM_BWD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    r, h = c.forward()
    o = c.backward(r)
    bufs = {k: torch.zeros_like(v) for k, v in o.items()}
    r2, h2 = torch.zeros_like(r), torch.zeros_like(h)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        P.moe_residual_norm(c.desc, c.norm, c.x, c.y, c.w_post, c.g, c.w_pre, r2, h2)
        P.moe_residual_norm_bwd(c.desc, c.norm, c.dr, c.dh, c.y, r2, c.w_post, c.g, c.w_pre, bufs["dx"], bufs["dy"],
                                bufs["dw_post"], bufs["dgate"], bufs["dw_pre"], ws, n)
    for k in range(3):
        c.x.copy_(torch.randn_like(c.x, dtype=torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        r, h = c.forward()
        o = c.backward(r)
        assert torch.equal(r, r2) and torch.equal(h, h2)
        assert all(torch.equal(o[k], bufs[k]) for k in o)
