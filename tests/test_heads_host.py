"""Host-side checks of the entry points for query and key heads (no GPU needed):
what they do before, or without, a launch."""
import os
import subprocess
import sys

import pytest

from paper_2603_13180_amd import mxnorm

pytestmark = pytest.mark.skipif(not os.path.exists(mxnorm.LIB_PATH), reason="libmxnorm.so not built")

# A backward call without heads and without gain gradients launches nothing, so its
# plan alone runs.  (In a process of its own: a plan that does not end is a failure
# here, not a test run that hangs.)
NO_HEADS = """
import ctypes, sys
I, L, P, F = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
class Heads(ctypes.Structure):
    _fields_ = [("data", P), ("heads", L), ("token_stride", L), ("head_stride", L)]
f = ctypes.CDLL(sys.argv[1]).qk_norm_rope_bwd
f.argtypes = [P] * 6 + [L] * 3 + [P, P, I, F] + [P] * 5 + [ctypes.c_size_t, P]
h = ctypes.byref(Heads(None, 0, 0, 0))
T, D, R = (int(a) for a in sys.argv[2:5])
sys.exit(f(h, h, h, h, None, None, T, D, R, None, 0x10000, 0, 1e-6, h, h, None, None, None, 0, None))
"""


@pytest.mark.parametrize("T,D,R", [(1, 64, 0), (8, 64, 0), (8, 64, 64), (4096, 512, 0), (1 << 40, 8, 0)])
def test_a_plan_without_heads_ends(T, D, R):
    run = [sys.executable, "-c", NO_HEADS, mxnorm.LIB_PATH, str(T), str(D), str(R)]
    assert subprocess.run(run, timeout=60).returncode == 0
