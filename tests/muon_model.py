"""The orthogonalised update in torch: by its definition in 64 bits, and with the roundings that the library states.

The library keeps X, its Gram matrix A and their polynomials in fp16, or in two fp16 parts, after powers of two that take values
of up to a matrix's bound to 2^14 .. 2^15, multiplies with fp32 sums, and takes steps together: two at first, then three (two in
the precise form) where the long side is 1.5 times the short one. Within a group, with P = a + b A + c A^2: Q <- P Q and A <- P (P A),
and X <- Q X ends it."""
import torch


def definition(u, eps, steps, coef, skip=0):
    """X in 64 bits. skip: steps left out."""
    a, b, c = coef
    flip = u.shape[0] > u.shape[1]
    x = u.double().t() if flip else u.double()
    x = x / (x.norm() + eps)
    for _ in range(steps - skip):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if flip else x


def most_of(f, top):
    """Largest |f| over [0, top] of a smooth function of few extrema."""
    t = torch.linspace(0.0, top, 20001, dtype=torch.float64)
    return float(f(t).abs().max())


def power_for(top):
    """The power of two that takes values of up to `top` into [2^14, 2^15)."""
    return 2.0 ** (14 - int(torch.floor(torch.log2(torch.tensor(max(top, 1e-6), dtype=torch.float64)))))


class Kept:
    """A matrix as it is kept: one or two fp16 parts of its values times a power of two."""

    def __init__(self, v, top, precise):
        self.s = power_for(top)
        w = (v * self.s).float()
        hi = w.half().float()
        self.parts = [hi, (w - hi).half().float()] if precise else [hi]

    def value(self):
        return sum(p.double() for p in self.parts) / self.s

    def t(self):
        k = object.__new__(Kept)
        k.s, k.parts = self.s, [p.t().contiguous() for p in self.parts]
        return k

    def __matmul__(self, o):
        """fp32 sums of the parts' products, the smallest left out."""
        out = self.parts[0] @ o.parts[0]
        if len(self.parts) == 2:
            out = (self.parts[0] @ o.parts[1] + self.parts[1] @ o.parts[0]) + out
        return out.double() / (self.s * o.s)


def rounded(u, eps, steps, coef, precise):
    """X with the library's roundings."""
    a, b, c = coef
    flip = u.shape[0] > u.shape[1]
    x = u.double().t() if flip else u.double()
    m, n = x.shape
    eye = torch.eye(m, dtype=torch.float64, device=x.device)
    top, done = 1.0, 0
    x = Kept(x / (x.norm() + eps), top, precise)
    while done < steps:
        group = min(steps - done, (2 if done == 0 or precise else 3) if 2 * n >= 3 * m else 1)
        A, Q, tq = Kept(x @ x.t(), top ** 2, precise), None, 1.0
        for i in range(group):
            tp = most_of(lambda t: a + b * t ** 2 + c * t ** 4, top)
            P = Kept(a * eye + b * A.value() + c * (A @ A), tp, precise)
            R = Kept(P @ A, tp * top ** 2, precise)
            tq *= tp
            Q = P if Q is None else Kept(P @ Q, tq, precise)
            top = most_of(lambda t: t * (a + b * t ** 2 + c * t ** 4), top)
            if i + 1 < group:
                A = Kept(P @ R, top ** 2, precise)
        done += group
        v = Q @ x
        if done == steps:
            return v.t() if flip else v
        x = Kept(v, top, precise)


def apart(x, y):
    return float((x.double() - y).norm() / y.norm())
