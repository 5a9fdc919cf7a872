"""What the norms between blocks, the 8-bit experts and the orthogonalised updates refuse, before any HIP call (no GPU is
touched)."""
import os

import pytest

from paper_2506_02965_amd import pcmoe as P

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libpcmoe.so not built")
OK = 0x1000        # an aligned address that is never followed: every call here is refused
INV, UNS, WS = P.MOE_ERR_INVALID_ARGUMENT, P.MOE_ERR_UNSUPPORTED, P.MOE_ERR_WORKSPACE_TOO_SMALL


def refused(status, fn, *args):
    with pytest.raises(P.MoeError) as e:
        fn(*args, stream=0)
    assert e.value.status == status, str(e.value)
    return str(e.value)


def desc(**kw):
    a = dict(T=64, d_model=256, d_ff=384, n_experts=16, top_k=4)
    a.update(kw)
    return P.make_desc(**a)


def norm(**kw):
    n = P.make_norm("rms", "rms", gate_groups=4)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


NORMS = [dict(pre=3), dict(post=-1), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
         dict(residual_scale=float("nan")), dict(residual_scale=float("inf")), dict(gate_groups=0), dict(gate_groups=-4),
         dict(gate_groups=5), dict(gate_groups=128)]


@pytest.mark.parametrize("kw", NORMS, ids=str)
def test_norm_settings(kw):
    d = desc()
    refused(INV, P.moe_residual_norm, d, norm(**kw), OK, OK, OK, OK, OK, OK, OK)
    refused(INV, P.moe_residual_norm_bwd, d, norm(**kw), *[OK] * 12, OK, 1 << 30)


def test_norm_arguments():
    d, n = desc(), norm()
    with pytest.raises(ValueError):
        P.make_norm("batch")
    # x, y, w_post, gate, w_pre, r, h
    for i in (0, 5, 6):
        for bad in (None, OK + 8):
            a = [OK] * 7
            a[i] = bad
            refused(INV, P.moe_residual_norm, d, n, *a)
    for i in (1, 2, 3, 4):
        a = [OK] * 7
        a[i] = OK + 4
        refused(INV, P.moe_residual_norm, d, n, *a)
    refused(INV, P.moe_residual_norm, d, norm(pre=0), OK, OK, OK, OK, OK, OK, None)     # w_pre without its norm
    refused(INV, P.moe_residual_norm, d, norm(pre=0), OK, OK, OK, OK, None, OK, OK)     # h without it
    refused(INV, P.moe_residual_norm, d, norm(post=0), OK, OK, OK, OK, OK, OK, OK)
    refused(INV, P.moe_residual_norm, d, norm(), OK, None, OK, OK, OK, None, OK)        # a post norm of nothing
    refused(INV, P.moe_residual_norm, d, norm(post=0), OK, None, None, OK, OK, None, OK)
    refused(INV, P.moe_residual_norm, d, norm(post=0, residual_scale=0.5), OK, None, None, None, OK, None, OK)
    refused(INV, P.moe_residual_norm, d, norm(post=0), OK, None, None, None, OK, OK, OK)     # r is x
    refused(INV, P.moe_residual_norm, d, norm(post=0, pre=0), OK, None, None, None, None, None, None)
    refused(UNS, P.moe_residual_norm, desc(d_model=200), n, *[OK] * 7)


def test_norm_bwd_arguments():
    d, n = desc(), norm()
    need = P.moe_workspace_size(d, P.MOE_WS_NORM_BWD)
    assert need > 0
    # dr, dh, y, r, w_post, gate, w_pre, dx, dy, dw_post, dgate, dw_pre, ws
    good = [OK] * 13
    for i in range(13):
        for bad in (None, OK + 8):
            if bad is None and i in (0, 4, 5, 6):     # dr and the weights may be absent (4..6 with their gradients)
                continue
            a = list(good)
            a[i] = bad
            refused(INV, P.moe_residual_norm_bwd, d, n, *a, need)
    for i in (4, 5, 6):        # the gradient of a weight that is not there
        a = list(good)
        a[i] = None
        refused(INV, P.moe_residual_norm_bwd, d, n, *a, need)
    refused(WS, P.moe_residual_norm_bwd, d, n, *good, need - 1)
    none = norm(pre=0)
    refused(INV, P.moe_residual_norm_bwd, d, none, None, None, OK, None, OK, OK, None, OK, OK, OK, OK, None, OK, need)
    refused(INV, P.moe_residual_norm_bwd, d, none, OK, OK, OK, None, OK, OK, None, OK, OK, OK, OK, None, OK, need)


def muon(**kw):
    o = P.make_muon()
    for k, v in kw.items():
        setattr(o, k, v)
    return o


MUONS = [(dict(lr=0.0), INV), (dict(lr=float("inf")), INV), (dict(momentum=1.0), INV), (dict(momentum=-0.1), INV),
         (dict(weight_decay=-0.1), INV), (dict(weight_decay=float("nan")), INV), (dict(scale=0.0), INV),
         (dict(scale=float("nan")), INV), (dict(eps=0.0), INV), (dict(steps=0), INV), (dict(steps=17), INV),
         (dict(nesterov=2), INV), (dict(precise=-1), INV), (dict(a=float("nan")), INV), (dict(c=float("inf")), INV),
         (dict(a=17.0, b=0.0, c=0.0), UNS), (dict(a=3.0, b=0.0, c=0.0), UNS), (dict(b=-40.0), UNS)]


@pytest.mark.parametrize("kw,status", MUONS, ids=str)
def test_muon_settings(kw, status):
    d = desc()
    for precise in (0, 1):
        refused(status, P.moe_expert_update_muon, d, muon(**{"precise": precise, **kw}), *[OK] * 9, 1 << 40)


def test_muon_arguments():
    for which, precise in ((P.MOE_WS_UPDATE_MUON, 0), (P.MOE_WS_UPDATE_MUON_PRECISE, 1)):
        d, o = desc(), muon(precise=precise)
        need = P.moe_workspace_size(d, which)
        good = [OK] * 9      # w_gate, w_up, w_down, dw_gate, dw_up, dw_down, master, m, ws
        for i in range(9):
            for bad in (None, OK + 8):
                if bad is None and i == 6:
                    continue
                a = list(good)
                a[i] = bad
                refused(INV, P.moe_expert_update_muon, d, o, *a, need)
        refused(WS, P.moe_expert_update_muon, d, o, *good, need - 1)
        refused(INV, P.moe_expert_update_muon, d, o, *good[:8], OK + 128, need)
    huge = desc(d_model=23296, d_ff=23296, n_experts=1, top_k=1)       # both parts of a matrix are one buffer
    refused(UNS, P.moe_expert_update_muon, huge, muon(precise=1), *[OK] * 9, 1 << 40)
    # X in both orientations and a turn of one, A and B, for three matrices of every expert
    assert P.moe_workspace_size(d, P.MOE_WS_UPDATE_MUON) >= 2 * 48 * (3 * 256 * 384 + 2 * 256 * 256)


def test_q8_pack_arguments():
    for fn, n_ptr in ((P.moe_q8_pack, 3), (P.moe_q8_unpack, 3)):
        for shape in ((0, 16, 128), (1, 0, 128), (1, 16, 0), (-1, 16, 128)):
            refused(INV, fn, *shape, "bf16", *[OK] * n_ptr)
        refused(UNS, fn, 1, 16, 64, "bf16", *[OK] * n_ptr)
        refused(UNS, fn, 1, 16, 200, "f32", *[OK] * n_ptr)
        refused(UNS, fn, 1 << 20, 1 << 20, 128, "bf16", *[OK] * n_ptr)
        for i in range(n_ptr):
            for bad in (None, OK + 8):
                a = [OK] * n_ptr
                a[i] = bad
                refused(INV, fn, 1, 7, 128, "bf16", *a)
        with pytest.raises(ValueError):
            fn(1, 16, 128, "f16", *[OK] * n_ptr, stream=0)


def test_ffn_q8_arguments():
    d = desc(n_shared=1)
    need = P.moe_workspace_size(d, P.MOE_WS_FFN_Q8)
    good = [OK] * 11       # x, x_perm, offsets, six of weights, y_perm, ws
    for i in range(11):
        for bad in (None, OK + 8):
            a = list(good)
            a[i] = bad
            refused(INV, P.moe_expert_ffn_q8, d, *a, need)
    refused(WS, P.moe_expert_ffn_q8, d, *good, need - 1)
    refused(UNS, P.moe_expert_ffn_q8, desc(n_shared=1, dtype="f32"), *good, need)
    assert P.moe_workspace_size(desc(dtype="f32"), P.MOE_WS_FFN_Q8) == 0
