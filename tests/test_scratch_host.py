"""Memory that the built library's kernels spill registers to, from the metadata of its code objects (no GPU is touched)."""
import os
import re
import struct
import subprocess

import pytest

from paper_2506_02965_amd import pcmoe as P

LLVM = "/opt/rocm/llvm/bin"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH) or not os.path.exists(f"{LLVM}/llvm-readelf"),
                                reason="needs the built library and llvm-readelf")


def code_objects(path):
    """The GPU code objects of a library: an offload bundle for each source file, a table of (offset, size, target) at its head."""
    data = open(path, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + len(MAGIC))
        o = at + len(MAGIC) + 8
        if n < 8:
            for _ in range(n):
                off, size, length = struct.unpack_from("<QQQ", data, o)
                target = data[o + 24:o + 24 + length]
                if target.endswith(b"gfx950") and size:
                    yield data[at + off:at + off + size]
                o += 24 + length
        at = data.find(MAGIC, at + 1)


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    """Bytes of scratch a lane by kernel."""
    out = {}
    file = tmp_path_factory.mktemp("co") / "co"
    for co in code_objects(P.LIB_PATH):
        file.write_bytes(co)
        text = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", str(file)], capture_output=True, text=True, check=True).stdout
        for kernel in text.split("- .agpr_count:")[1:]:
            name = re.search(r"^\s*\.name:\s*(\S+)", kernel, re.M).group(1)
            out[name] = int(re.search(r"\.private_segment_fixed_size:\s*(\d+)", kernel).group(1))
    return out


def test_norms(scratch):
    """Rows of any length: the longest once spilled up to 3.7 KB a lane, and took ten times their bytes' time."""
    norms = {k: v for k, v in scratch.items() if "residual_norm" in k}
    assert len(norms) > 40
    assert max(norms.values()) <= 64, {k: v for k, v in norms.items() if v > 64}
