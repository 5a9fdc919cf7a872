"""The workgroups of the 8-bit experts that walk over several tiles, and rows of every kind of tile, against 64 bits and each other.

`tiles_of` and `kind` repeat the library's choice of tiles and their order, so that each test knows what it reaches: that workgroups
take a second and a third tile, go from whole tiles to partial ones and to tails, and from tail to tail."""
import math

import pytest
import torch

from test_gpu_q8 import Experts

pytestmark = pytest.mark.gpu
CUS = 256


def kind(T, d, f, E, k, S, down):
    """'few' (64 rows), 'mid' (128) or 'large' (256, the walking kernel)."""
    mean = (T * k + T * S) / (E + S)

    def expected(bm):
        return (E + S) * (mean / bm + 0.5)
    kts, n = (f if down else d) / 128, d if down else 2 * f
    large, mid = expected(256) * math.ceil(n / 256), expected(128) * math.ceil(n / 128)
    if mean < 64 or mid <= CUS:
        return "few"
    return "large" if math.ceil(large / CUS) * (1.55 * kts + 10) <= math.ceil(mid / (2 * CUS)) * (1.15 * kts + 3) else "mid"


def walks(counts, T, d, f, S, down):
    """For each workgroup the kinds of its tiles in order: 'full' and 'part' of 256 rows, 'tail' of 128."""
    nt = (d + 255) // 256 if down else f // 128
    body, tails = [], []
    for rows in list(counts) + [T] * S:
        rem = rows % 256
        tail = 0 < rem <= 128
        tiles = -(-rows // 256) - tail
        kinds = ["full"] * (rows // 256) + (["part"] if rem > 128 else [])
        for b in range(0, tiles, 8):        # bunches of eight m-tiles for each n-tile
            bunch = kinds[b:b + 8]
            body += bunch * nt
        tails += ["tail"] * (tail * nt)
    out = []
    for x in range(8):
        mine = []
        for l in (body, tails):
            q, r = divmod(len(l), 8)
            at = x * q + min(x, r)
            mine += l[at:at + q + (x < r)]
        out += [mine[w::CUS // 8] for w in range(CUS // 8)]
    return out


def steps(w):
    return {(a, b) for seq in w for a, b in zip(seq, seq[1:])}


KINDS = ("full", "part", "tail")
# steps from one tile to the next: whole tiles come before tails
ALL = {(a, b) for a in KINDS for b in KINDS if a != "tail" or b == "tail"}
# T, d, f, rows of the experts, shared experts, the projection whose workgroups take several tiles, the steps that it must hold
CASES = [
    (1177, 1024, 8192, [138, 254, 397, 178, 101, 109], 0, "gate_up", ALL - {("tail", "tail")}),
    (3760, 1024, 2816, [620, 326, 36, 308, 306, 11, 71, 41, 124, 922, 250, 59, 75, 100, 302, 209], 0, "gate_up", ALL),
    (4558, 8192, 1024, [557, 612, 17, 236, 1105, 32, 16, 1016, 45, 74, 11, 837], 0, "down", ALL),
    (2500, 2048, 2816, [1281, 900, 60, 259], 1, "gate_up", {("full", "full"), ("full", "part"), ("part", "full"), ("full", "tail")}),
    (6000, 4096, 4096, [5000, 127, 300, 573], 0, "gate_up and down", {("full", "full"), ("full", "tail")}),
]


@pytest.mark.parametrize("T,d,f,counts,S,which,want", CASES)
def test_workgroups_that_take_several_tiles(T, d, f, counts, S, which, want):
    assert torch.cuda.get_device_properties(0).multi_processor_count == CUS
    for name, down in (("gate_up", False), ("down", True)):
        if name in which:
            assert kind(T, d, f, len(counts), 1, S, down) == "large"
            w = walks(counts, T, d, f, S, down)
            assert sum(len(s) for s in w) > CUS and want <= steps(w), steps(w)
    e = Experts(T, d, f, len(counts), 1, S, counts=counts)
    y = e.check()
    assert torch.equal(e.run(), y)


@pytest.mark.parametrize("T,d,f,kinds", [(4000, 2048, 1024, ("large", "large")), (2560, 2048, 1024, ("mid", "mid"))])
def test_rows_in_large_and_small_calls(T, d, f, kinds):
    """Rows of 128- and 256-row tiles are those of 64-row tiles in calls of their own."""
    counts = [1300, T - 1300]
    assert (kind(T, d, f, 2, 1, 0, False), kind(T, d, f, 2, 1, 0, True)) == kinds
    e = Experts(T, d, f, 2, 1, counts=counts)
    y = e.run()
    for first, n in ((0, 1), (200, 60), (1250, 50), (1300, 17), (2500, 60)):
        g = int(first >= 1300)
        assert kind(n, d, f, 2, 1, 0, False) == kind(n, d, f, 2, 1, 0, True) == "few"
        s = Experts(n, d, f, 2, 1, counts=[n, 0] if g == 0 else [0, n])
        s.gate, s.up, s.down = e.gate, e.up, e.down
        s.x_perm = e.x_perm[first:first + n].clone()
        assert torch.equal(s.run()[:n], y[first:first + n]), (first, n)
