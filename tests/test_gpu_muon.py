"""moe_expert_update_muon against 64 bits.

Tolerances are on the 2-norm of an update matrix. With u the relative rounding of every matrix that is kept (2^-11, half a
step of fp16; 2^-21 where each is held in two parts) and products that sum K terms in fp32 (K / 16 + 8 roundings of 2^-24),
errors are followed to first order through the products that the library takes: A = X X^T, and for the steps of a group (two
steps, then three at a time, or two in the precise form, where the long side is 1.5 times the short one; else every step
alone) P = a + b A + c A^2,
Q <- P Q, and between steps R = P A, A <- P R; then X <- Q X. An error of X itself is passed on by at most slope = |p'| (or the
largest quotient of differences), which a bounds, for each step. All of it is formed from the 64-bit run itself."""
import pytest
import torch

from paper_2506_02965_amd import pcmoe as P

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)
U32 = 2.0 ** -24


def groups(m, n, steps, precise):
    first = True
    while steps > 0:
        g = min(steps, (2 if first or precise else 3) if 2 * n >= 3 * m else 1)
        yield g
        steps -= g
        first = False


def orthogonalise(u, eps, steps, coef, unit):
    """X after the steps in 64 bits, and a bound of the 2-norm (Frobenius) of what rounding does to it."""
    a, b, c = coef
    flip = u.shape[0] > u.shape[1]
    x = (u.t() if flip else u).contiguous()
    x = x / (x.norm() + eps)
    m, n = x.shape
    eye = torch.eye(m, dtype=torch.float64, device=x.device)
    # every matrix is a polynomial of X: its largest singular value is that of X's singular values
    s = torch.linalg.svdvals((x @ x.t()).cpu()).clamp(min=0).sqrt()

    def two(v):
        return float(v.abs().max())

    def kept(t, v, terms):
        """Rounding of a product of `terms` terms that is kept: its own, and its sums' (their absolute terms in `terms[1]`).
        Elements below fp16's normal range (numbers scaled to 2^14 at least) are off by 2^-25 of that scale at most."""
        k, size = terms
        return unit * float(t.norm()) + (k / 16 + 8) * U32 * size + 2.0 ** -39 * t.numel() ** 0.5 * max(1.0, two(v))
    slope = max(abs(a), 2.0)
    err = kept(x, s, (0, 0.0))
    for g in groups(m, n, steps, unit < 2.0 ** -20):
        gram, l = x @ x.t(), s ** 2
        e_a = kept(gram, l, (n, float(x.norm()) ** 2))
        q, v, e_q = eye, torch.ones_like(s), 0.0
        for i in range(g):
            p, w = a * eye + b * gram + c * gram @ gram, a + b * l + c * l ** 2
            e_p = (abs(b) + 2 * abs(c) * two(l)) * e_a + kept(p, w, (m, abs(c) * float(gram.norm()) ** 2))
            if i == 0:
                new_q, e_q = p, e_p
            else:
                new_q = p @ q
                e_q = two(w) * e_q + two(v) * e_p + kept(new_q, w * v, (m, float(p.norm() * q.norm())))
            if i + 1 < g:
                r = p @ gram
                e_r = two(w) * e_a + two(l) * e_p + kept(r, w * l, (m, float(p.norm() * gram.norm())))
                new = p @ r
                e_a = two(w) * e_r + two(w * l) * e_p + kept(new, w * w * l, (m, float(p.norm() * r.norm())))
                gram, l = new, w * w * l
            q, v = new_q, v * w
        new = q @ x
        err = slope ** g * err + two(s) * e_q + kept(new, s * v, (m, float(q.norm() * x.norm()))) + 4 * U32 * float(new.norm())
        x, s = new, s * v
    return (x.t() if flip else x), float(err)


class Run:
    def __init__(self, d, f, E, shared=0, dtype="bf16", master=False, seed=0, local=None, **opt):
        self.G = (E if local is None else local) + shared
        self.d, self.f, self.dt = d, f, torch.bfloat16 if dtype == "bf16" else torch.float32
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + d + 31 * f)
        self.sides = ((f, d), (f, d), (d, f))

        def normal(*s, std=1.0, dtype=None):
            return (torch.randn(*s, device="cuda", generator=g) * std).to(dtype or self.dt)
        self.w = [normal(self.G, a, b, std=b ** -0.5) for a, b in self.sides]
        self.g = [normal(self.G, a, b, std=1e-3) for a, b in self.sides]
        self.m = normal(3 * self.G * f * d, std=2e-3, dtype=torch.float32)
        self.master = torch.cat([t.reshape(-1).float() for t in self.w]) + 1e-5 if master else None
        o = dict(lr=0.02, momentum=0.95, weight_decay=0.1, scale=0.2 * max(d, f) ** 0.5, coefficients=COEF)
        o.update(opt)
        self.opt = P.make_muon(**o)
        self.desc = P.make_desc(1, d, f, max(E, 1), 1, 0, local, shared, dtype=dtype)
        which = P.MOE_WS_UPDATE_MUON_PRECISE if self.opt.precise else P.MOE_WS_UPDATE_MUON
        self.ws = torch.empty(P.moe_workspace_size(self.desc, which), dtype=torch.uint8, device="cuda")

    def step(self):
        P.moe_expert_update_muon(self.desc, self.opt, *self.w, *self.g, self.master, self.m, self.ws, self.ws.numel())

    def state(self):
        return [t.clone() for t in (*self.w, self.m)] + ([] if self.master is None else [self.master.clone()])

    def check(self):
        o = self.opt
        w0, m0 = [t.clone() for t in self.w], self.m.clone()
        p0 = None if self.master is None else self.master.clone()
        self.step()
        n = self.d * self.f
        unit = 2.0 ** -21 if o.precise else 2.0 ** -11
        for t in range(3):
            for i in range(self.G):
                at = (t * self.G + i) * n
                shape = self.sides[t]
                old, g = m0[at:at + n].view(shape).double(), self.g[t][i].double()
                m = float(o.momentum) * old + g
                got = self.m[at:at + n].view(shape).double()
                tol = 2 * U32 * (old.abs() + g.abs())
                assert ((got - m).abs() <= tol).all()
                u = g + float(o.momentum) * got if o.nesterov else got
                x, err = orthogonalise(u, float(o.eps), o.steps, (float(o.a), float(o.b), float(o.c)), unit)
                err += 4 * U32 * float(x.norm())        # u and its norm
                p = w0[t][i].double() if p0 is None else p0[at:at + n].view(shape).double()
                want = p * (1 - float(o.lr) * float(o.weight_decay)) - float(o.lr) * float(o.scale) * x
                bound = float(o.lr) * float(o.scale) * err + 4 * U32 * float(p.norm() + want.norm())
                if p0 is not None:
                    new = self.master[at:at + n].view(shape)
                    assert float((new.double() - want).norm()) <= bound, (t, i)
                    assert torch.equal(self.w[t][i], new.to(self.dt))
                else:
                    off = float((self.w[t][i].double() - want).norm())
                    bound += torch.finfo(self.dt).eps / 2 * float(want.norm() + bound)
                    assert off <= bound, (t, i, off, bound)


SIZES = [(128, 128, 1), (128, 384, 2), (384, 128, 1), (256, 640, 3), (640, 256, 1), (512, 512, 2), (1024, 384, 1),
         (1408, 256, 1)]


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,f,E", SIZES)
def test_update(d, f, E, dtype, precise):
    Run(d, f, E, dtype=dtype, precise=precise).check()


@pytest.mark.parametrize("opt", [dict(steps=1), dict(steps=2), dict(steps=9), dict(nesterov=False), dict(momentum=0.0),
                                 dict(weight_decay=0.0), dict(coefficients=(1.5, -0.5, 0.0)), dict(coefficients=(2.0, -1.5, 0.5)),
                                 dict(coefficients=(1.0, 0.0, 0.0)), dict(eps=0.5)], ids=str)
@pytest.mark.parametrize("precise", [False, True])
def test_settings(opt, precise):
    Run(256, 384, 2, shared=1, precise=precise, **opt).check()


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_master_copy_and_shards(dtype, precise):
    Run(384, 256, 8, shared=1, local=3, dtype=dtype, master=True, precise=precise).check()


def test_larger_matrices():
    """Several tiles of every size each way, and many matrices in one launch."""
    Run(1024, 1280, 2, dtype="bf16").check()
    Run(640, 2176, 1, dtype="f32", precise=True).check()
    Run(256, 256, 24, dtype="bf16").check()


@pytest.mark.parametrize("d,f,E,dtype,precise", [(1024, 1536, 9, "bf16", False), (1536, 1024, 9, "f32", True),
                                                 (640, 896, 16, "bf16", True), (896, 640, 16, "f32", False)])
def test_large_tiles_and_their_quarters(d, f, E, dtype, precise):
    """So many matrices that the 256 x 256 tiles are taken: 270 of them on and above the diagonals, the last 14 in quarters, and
    288 of matrices that end within a tile."""
    Run(d, f, E, dtype=dtype, precise=precise).check()


@pytest.mark.parametrize("d,f,E,dtype,precise", [(128, 2048, 1, "f32", True), (4096, 128, 2, "bf16", False), (256, 3200, 2, "bf16", True),
                                                 (2176, 384, 1, "bf16", False), (128, 1152, 8, "f32", False)])
def test_long_rows_split_their_sums(d, f, E, dtype, precise):
    """Matrices of few rows and long columns, whose Gram matrices are summed in parts."""
    Run(d, f, E, dtype=dtype, precise=precise).check()


def test_zero_tiny_huge_and_broken_gradients():
    for precise in (False, True):
        r = Run(256, 384, 6, precise=precise, dtype="f32")
        n = r.d * r.f
        for t in range(3):
            for i, k in enumerate((0.0, 1e-25, 1e25)):
                r.g[t][i] *= k
                r.m[(t * 6 + i) * n:(t * 6 + i + 1) * n] *= k
            r.g[t][4][3, 5] = float("nan")
            r.g[t][5][100, 7] = float("inf")
        before = [w.clone() for w in r.w]
        r2 = Run(256, 384, 6, precise=precise, dtype="f32")      # the same without the broken ones
        r.step()
        r2.step()
        for t in range(3):
            keep = before[t][0].double() * (1 - float(r.opt.lr) * float(r.opt.weight_decay))
            assert ((r.w[t][0].double() - keep).abs() <= 2 * U32 * keep.abs()).all()      # nothing to follow
            for i in (1, 2):     # the direction does not depend on the size (1e-25: its norm is near eps, 1e25: it is far)
                assert torch.isfinite(r.w[t][i]).all()
            gone = 0.02 * float(r.opt.scale)
            off = (r.w[t][2] - r2.w[t][2]).norm() / gone
            # both runs round X apart: twice the bound of one
            _, err = orthogonalise(r2.g[t][2].double() + 0.95 * r2.m[(t * 6 + 2) * n:(t * 6 + 3) * n].view(r.sides[t]).double(),
                                   1e-7, 5, COEF, 2.0 ** -21 if precise else 2.0 ** -11)
            assert float(off) <= 2 * err + 1e-5 * float(r2.w[t][2].norm()) / gone
            assert torch.equal(r.w[t][3], r2.w[t][3])     # no other matrix is touched by a broken one
            assert torch.isnan(r.w[t][4]).all() and torch.isnan(r.w[t][5]).all()


def test_many_steps_make_singular_values_alike():
    """The definition's purpose: of a full-rank update every singular value ends between 0.6 and 1.25 (the range into which the
    polynomial takes values of 0.003 and more in five steps)."""
    r = Run(256, 256, 1, dtype="f32", precise=True, weight_decay=0.0, lr=1.0, scale=1.0)
    for t in range(3):
        q, _ = torch.linalg.qr(torch.randn(256, 256, device="cuda", dtype=torch.float64))
        v, _ = torch.linalg.qr(torch.randn(256, 256, device="cuda", dtype=torch.float64))
        s = torch.linspace(0.05, 1.0, 256, device="cuda", dtype=torch.float64)
        r.g[t][0] = (q * s @ v).float()
    r.m.zero_()
    before = [w.clone() for w in r.w]
    r.step()
    for t in range(3):
        s = torch.linalg.svdvals((before[t][0] - r.w[t][0]).double())
        assert 0.6 < float(s.min()) and float(s.max()) < 1.25


def test_equal_calls_and_graph_replays():
    a, b = Run(256, 384, 2, seed=4), Run(256, 384, 2, seed=4)
    a.step()
    b.step()
    assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.step()
    for k in range(3):
        for t in range(3):
            new = torch.randn_like(a.g[t], dtype=torch.float32) * 1e-3
            a.g[t].copy_(new)
            b.g[t].copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        a.step()
        assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state())), k


def test_nothing_behind_the_workspace_or_state_is_written():
    r = Run(128, 256, 2)
    guard = 4096
    for name in ("ws", "m"):
        t = getattr(r, name)
        pad = guard // t.element_size()
        whole = torch.full((t.numel() + pad,), 3, dtype=t.dtype, device="cuda")
        whole[:t.numel()].copy_(t)
        setattr(r, name + "_whole", whole)
        setattr(r, name, whole[:t.numel()])
    r.check()
    assert (r.ws_whole[r.ws.numel():] == 3).all() and (r.m_whole[r.m.numel():] == 3).all()


def test_matrices_taken_in_several_passes():
    """Small matrices of so many experts that the workspace holds some of them at a time: 1,032 of 256 x 128, and 96 of 640 x 256
    (six tiles each), as the matrices alone would be."""
    for d, f, E, dtype, picks in ((128, 256, 256, "bf16", (0, 100, 255)), (256, 640, 256, "f32", (0, 200))):
        r = Run(d, f, E, shared=88 if d == 128 else 0, dtype=dtype, master=True)
        n, G = d * f, r.G
        alone = Run(d, f, len(picks), dtype=dtype, master=True)
        for t in range(3):
            for k, i in enumerate(picks):
                alone.w[t][k], alone.g[t][k] = r.w[t][i], r.g[t][i]
                for name in ("m", "master"):
                    getattr(alone, name)[(t * len(picks) + k) * n:][:n] = getattr(r, name)[(t * G + i) * n:][:n]
        r.step()
        alone.check()       # against 64 bits
        for t in range(3):
            for k, i in enumerate(picks):
                # other tiles may add up in another order
                a = alone.master[(t * len(picks) + k) * n:][:n]
                b = r.master[(t * G + i) * n:][:n]
                assert float((a - b).norm()) <= 0.02 * float(r.opt.lr) * float(r.opt.scale) * min(d, f) ** 0.5
