"""What the norm kernel's device code promises about the alignment of rows: no more than an element's (CPU only)."""
import os
import re
import subprocess

import pytest

from paper_1712_01084_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows_of_any_alignment(tmp_path):
    """Rows may start at any element: wide loads from global memory are declared to need 2 or 4 bytes of alignment, and wide
    stores 1 to 4."""
    try:
        hipcc = build._hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    out = str(tmp_path / "norm.ll")
    flags = [f for f in build.DEVICE if f != "--offload-compress"]
    cmd = [hipcc] + build.COMMON + flags + ["--cuda-device-only", "-S", "-emit-llvm", os.path.join(build.CSRC, "pivot_norm.hip"), "-o", out]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]
    wide = re.findall(r"= load <(\d+) x (\w+)>, ptr addrspace\(1\) [^,]+, align (\d+)", open(out).read())
    size = {"i8": 1, "i16": 2, "half": 2, "i32": 4, "float": 4, "i64": 8, "double": 8}
    wide = [(int(n) * size[t], int(a)) for n, t, a in wide]
    assert any(b == 16 for b, _ in wide)
    assert all(a <= 4 for b, a in wide if b >= 8), sorted(set(wide))
