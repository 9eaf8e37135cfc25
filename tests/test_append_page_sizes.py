"""Host side of the E4M3 append calls at page sizes up to the largest number: the calls return."""
import os
import subprocess
import sys

import pytest

from paper_2605_15250_b200 import build as gbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALL = """
import ctypes, sys
from paper_2605_15250_b200 import binding as B
P, d = ctypes.c_void_p(0x1000), ctypes.byref(B.make_dims(128, 8, 128, 512, 64))
front, mid = [d, 0, 2, 5, P, P], [P, 64, P, 100, 0, None, 0, 0, None, 0, 0]
page = int(sys.argv[2])
if sys.argv[1] == "latent":
    code = B.lib().gqla_append_rope_fp8(*front, P, 512, *mid, P, 576, 640, P, P, 4, page, None, None)
else:
    code = B.lib().gqla_append_planes_fp8(*front, P, P, *mid, P, P, P, 64, 640, P, P, P, P, 4, page, None, None)
print("code", code)
"""


@pytest.mark.parametrize("page", [1, 3, 64, 1 << 29, (1 << 30) - 1, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("call", ["latent", "planes"])
def test_append_returns_at_every_page_size(call, page):
    """In a process that sees no GPU: everything up to the launch runs, which then fails (6, GQLA_ERR_CUDA)."""
    gbuild.build()
    res = subprocess.run([sys.executable, "-c", CALL, call, str(page)], cwd=ROOT, timeout=120, capture_output=True, text=True,
                         env={**os.environ, "CUDA_VISIBLE_DEVICES": "", "PYTHONPATH": ROOT})
    assert res.returncode == 0 and res.stdout.split() == ["code", "6"], (res.stdout, res.stderr)
