"""bf16 outputs of the experts with 4-bit weights are the sums rounded once, whatever the size of the call.

What stands between the fp64 result and the rounding: H as two bf16 numbers (2^-17 of each value), its fp32 sums, exponential
and reciprocal (2^-20), the fp32 sums over K (2^-20). Over independent terms that is less than d = 1e-5 of the outputs' norm
per root of their number. An output rounds otherwise where a rounding boundary lies within its error; boundaries lie 2^-8 to
2^-7 of the output apart, so among normally distributed outputs at most about sqrt(2/pi) a (1 + ln(1/a)) = 1.4% do, a = 2^8 d.
4% are allowed. (H rounded to bf16 alone: d = 1.6e-3, and a third of them.)"""
import pytest
import torch

from gpu_util import log
from test_gpu_q4 import run

pytestmark = pytest.mark.gpu

CASES = [  # T, d, f, rows per hosted expert, k, E, shared, group
    (1, 1152, 1408, [0, 1], 1, 2, 2, 128),                        # K split over the wavefronts
    (9, 4096, 1024, [9, 4, 5], 2, 3, 0, 64),
    (24, 4096, 1792, [24, 3, 21], 2, 3, 0, 64),                   # a decode batch
    (60, 384, 512, [20, 17, 33, 16, 1, 33], 2, 6, 0, 32),         # 16-row chunks
    (100, 640, 384, [50, 49, 97, 4], 2, 4, 1, 32),
    (800, 640, 384, [200, 129, 31, 33, 800, 0, 7, 400], 2, 8, 0, 32),   # 32 rows x 128 columns
    (777, 1024, 2816, [777, 400, 377], 2, 3, 0, 32),              # a prompt
    (40, 128, 128, [9, 0, 12], 4, 12, 0, 32),                     # K of one and two steps, up to 16 rows and more
    (70, 640, 256, [5, 70, 64, 1], 2, 4, 0, 64),
    (300, 256, 128, [300, 150, 150], 2, 3, 1, 128),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "T{}_d{}_f{}_g{}".format(c[0], c[1], c[2], c[7]))
def test_outputs_are_rounded_once(case):
    T, d, f, counts, k, E, S, group = case
    log(f"[q4] rounding {case}")
    y, ref, valid, _ = run(T, d, f, counts, k, E, S, group, "bf16")
    off = float((y[valid] != ref[valid].bfloat16().double()).double().mean())
    log(f"[q4] rounding {off:.4f} of the outputs differ from the rounded fp64 result")
    assert off <= 0.04, off


@pytest.mark.parametrize("hosted,shared", [(256, 70), (256, 255), (3, 317)])
def test_more_than_256_groups(hosted, shared):
    """Hosted and shared experts together, up to the most that a call takes; most of them without a row."""
    T, k = 2, 4
    counts = [0] * hosted
    for g in (0, hosted // 2, hosted - 1):
        counts[g] = 2
    log(f"[q4] groups {hosted} + {shared}")
    y, ref, valid, _ = run(T, 128, 128, counts, min(k, hosted), 256, shared, 64, "bf16")
    off = float((y[valid] != ref[valid].bfloat16().double()).double().mean())
    assert off <= 0.04 and bool((y[~valid] == 77).all()), off
