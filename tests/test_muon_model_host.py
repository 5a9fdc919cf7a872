"""The model that the GPU's orthogonalised updates are held against: how far its roundings take X from the definition, and that the
allowed distance (three times that) excludes what is wrong. Random matrices as in the GPU tests."""
import pytest
import torch

from muon_model import apart, definition, rounded

COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def matrix(m, n):
    g = torch.Generator().manual_seed(m + 31 * n)
    return torch.randn(m, n, generator=g) * 1e-3


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("m,n,steps", [(128, 128, 5), (128, 384, 5), (384, 128, 5), (256, 384, 9), (512, 512, 5), (1024, 1536, 5),
                                       (128, 2048, 5)])
def test_the_allowed_distance_excludes_errors(m, n, steps, precise):
    u = matrix(m, n)
    x = definition(u, EPS, steps, COEF)
    allowed = 3 * apart(rounded(u, EPS, steps, COEF, precise), x)
    assert allowed < (2e-5 if precise else 1e-2)
    wrong = {"nothing": 0 * x, "the other way": -x, "a step less": definition(u, EPS, steps, COEF, skip=1),
             "a step more": definition(u, EPS, steps + 1, COEF),
             "transposed": definition(u.t().contiguous(), EPS, steps, COEF).reshape(x.shape)}
    for k in range(3):
        wrong[f"coefficient {k} 1% off"] = definition(u, EPS, steps, tuple(v * 1.01 if i == k else v for i, v in enumerate(COEF)))
    for name, v in wrong.items():
        if name == "transposed" and m == n:
            continue
        assert apart(v, x) > 2 * allowed, name


def test_the_model_without_roundings_is_the_definition(monkeypatch):
    """Groups of steps are the steps."""
    import muon_model
    monkeypatch.setattr(muon_model, "power_for", lambda top: 1.0)
    monkeypatch.setattr(torch.Tensor, "half", lambda t: t)
    monkeypatch.setattr(torch.Tensor, "float", lambda t: t)
    for m, n in ((128, 384), (128, 160)):
        for precise in (False, True):
            u = matrix(m, n).double()
            assert apart(rounded(u, EPS, 6, COEF, precise), definition(u, EPS, 6, COEF)) < 1e-9
