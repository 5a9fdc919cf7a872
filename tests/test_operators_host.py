"""What the gated routing, the 8-bit checkpoints and the 4-bit experts refuse, before any HIP call (no GPU is touched)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_02965_amd import pcmoe as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


GATES = [
    (dict(n_groups=3), INV), (dict(n_groups=0), INV), (dict(n_groups=-4), INV), (dict(n_groups=4, topk_groups=5), INV),
    (dict(n_groups=4, topk_groups=0), INV), (dict(n_groups=8, topk_groups=1), INV), (dict(group_top=3), INV),
    (dict(group_top=0), INV), (dict(n_groups=16, topk_groups=8, group_top=2), INV), (dict(scale=0.0), INV),
    (dict(scale=-1.0), INV), (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV),
]


@pytest.mark.parametrize("kw,status", GATES, ids=lambda v: str(v))
def test_gate_settings(kw, status):
    g = P.make_gate(**kw)
    refused(status, P.moe_route_gated, desc(), g, OK, OK, None, 1, None, OK, OK, OK)
    refused(status, P.moe_route_gated_bwd, desc(), g, OK, OK, OK, OK, OK, OK, OK, OK, 1 << 40)


def test_subnormal_scale_has_no_reciprocal():
    refused(INV, P.moe_route_gated, desc(), P.make_gate(scale=1e-39), OK, OK, None, 1, None, OK, OK, OK)
    refused(INV, P.moe_route_gated_bwd, desc(), P.make_gate(scale=1e-39), OK, OK, OK, OK, OK, OK, OK, OK, 1 << 40)


def test_more_groups_than_lanes():
    refused(UNS, P.moe_route_gated, desc(n_experts=256), P.make_gate(n_groups=128, topk_groups=128), OK, OK, None, 1, None,
            OK, OK, OK)


def test_gate_kind():
    with pytest.raises(ValueError):
        P.make_gate("tanh")
    g = P.make_gate()
    g.score = 2
    refused(INV, P.moe_route_gated, desc(), g, OK, OK, None, 1, None, OK, OK, OK)
    st = P.lib().moe_route_gated(ctypes.byref(desc()), None, OK, OK, None, 1, None, OK, OK, OK, None)
    assert st == INV and "gate is NULL" in P.last_error()


def test_route_gated_pointers():
    good = [OK, OK, None, 1, None, OK, OK, OK]
    for i in (0, 1, 5, 6, 7):
        for bad in (None, OK + 4):
            a = list(good)
            a[i] = bad
            refused(INV, P.moe_route_gated, desc(), P.make_gate(), *a)
    refused(INV, P.moe_route_gated, desc(), P.make_gate(), OK, OK, None, 1, OK + 2, OK, OK, OK)
    refused(INV, P.moe_route_gated, desc(), P.make_gate(), OK, OK, OK, 3, None, OK, OK, OK)
    refused(INV, P.moe_route_gated, desc(top_k=17), P.make_gate(), *good)


def test_route_gated_bwd_pointers_workspace_and_shards():
    need = P.moe_workspace_size(desc(), P.MOE_WS_ROUTE_BWD)
    good = [OK] * 8
    for i in range(7):
        for bad in (None, OK + 8):
            a = list(good)
            a[i] = bad
            refused(INV, P.moe_route_gated_bwd, desc(), P.make_gate(), *a, need)
    refused(WS, P.moe_route_gated_bwd, desc(), P.make_gate(), *good, need - 1)
    refused(INV, P.moe_route_gated_bwd, desc(), P.make_gate(), *good[:7], OK + 16, need)
    msg = refused(INV, P.moe_route_gated_bwd, desc(local_begin=0, local_count=4), P.make_gate(), *good, need)
    assert "moe_route_gated_bwd needs every expert" in msg


@pytest.mark.parametrize("dtype,es", [("bf16", 2), ("f32", 4)])
def test_checkpoint_size_and_refusals(dtype, es):
    d = desc(dtype=dtype, n_shared=2)
    rows = 64 * (4 + 2)
    saved, need = P.moe_workspace_size(d, P.MOE_WS_FFN_SAVED), P.moe_workspace_size(d, P.MOE_WS_FFN_CKPT)
    rest = saved - rows * 384 * 3 * es                    # the plan (row counts are multiples of 256 bytes here)
    assert need == rows * 2 * 384 + rows * 2 * 384 // 32 + rest
    refused(WS, P.moe_ffn_checkpoint, d, OK, OK, OK, need - 1)
    refused(WS, P.moe_ffn_restore, d, OK, OK, need - 1, OK)
    for i in range(3):
        for bad in (None, OK + 8):
            a = [OK, OK, OK]
            a[i] = bad
            refused(INV, P.moe_ffn_checkpoint, d, *a, need)
            refused(INV, P.moe_ffn_restore, d, a[0], a[2], need, a[1])


SHAPES = [((0, 16, 128, 32, "bf16"), INV), ((1, 0, 128, 32, "bf16"), INV), ((1, 16, -128, 32, "bf16"), INV),
          ((1, 16, 128, 16, "bf16"), INV), ((1, 16, 128, 96, "f32"), INV), ((1, 24, 128, 32, "bf16"), UNS),
          ((1, 16, 192, 64, "bf16"), UNS), ((1 << 12, 1 << 14, 1 << 14, 32, "bf16"), UNS)]


@pytest.mark.parametrize("shape,status", SHAPES, ids=lambda v: str(v))
def test_q4_shapes(shape, status):
    refused(status, P.moe_q4_pack, *shape, OK, OK, OK)
    refused(status, P.moe_q4_unpack, *shape, OK, OK, OK)


def test_q4_pointers_and_workspace():
    for i in range(3):
        for bad in (None, OK + 8):
            a = [OK, OK, OK]
            a[i] = bad
            refused(INV, P.moe_q4_pack, 1, 16, 128, 32, "bf16", *a)
            refused(INV, P.moe_q4_unpack, 1, 16, 128, 32, "bf16", *a)
    d = desc(n_shared=1)
    need = P.moe_workspace_size(d, P.MOE_WS_FFN_Q4)
    assert need >= 64 * 5 * 384 * 2             # H, and room for its second part
    good = [OK] * 11
    for i in range(10):
        for bad in (None, OK + 8):
            a = list(good)
            a[i] = bad
            refused(INV, P.moe_expert_ffn_q4, d, 32, *a, need)
    refused(WS, P.moe_expert_ffn_q4, d, 32, *good, need - 1)
    refused(INV, P.moe_expert_ffn_q4, d, 48, *good, need)
    refused(INV, P.moe_expert_ffn_q4, d, 32, *good[:10], OK + 16, need)


def test_exports_every_declared_symbol():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pcmoe_ext.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"^\s*moe_status\s+(moe_\w+)\s*\(", src, flags=re.M)))
    assert sorted(P.EXPORTS_EXT) == names
    assert all(hasattr(P.lib(), n) for n in names)


def test_header_compiles_as_c(tmp_path):
    if shutil.which("gcc") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("gcc or the ROCm headers are not available")
    src = tmp_path / "ext_check.c"
    src.write_text('#include "pcmoe_ext.h"\n'
                   "int main(void) {\n"
                   "  moe_desc d = {0};\n"
                   "  moe_gate g = {MOE_SCORE_SIGMOID, 1, 1, 1, 1.0f};\n"
                   "  return moe_route_gated(&d, &g, 0, 0, 0, 1, 0, 0, 0, 0, 0) == MOE_OK ? MOE_NO_EXPERT : 0;\n"
                   "}\n")
    r = subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-fsyntax-only", "-D__HIP_PLATFORM_AMD__",
                        "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), str(src)],
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "pcmoe_ext.h" not in r.stderr, r.stderr
