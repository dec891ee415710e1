"""A launch that fails is the last one of its call (no GPU needed: without a device every launch fails).  The kernels behind it would
take what it has not written as indices."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (in a process without a device, so that nothing is launched on a machine that has one)
_ROUTE = """
import ctypes as C
import paper_1904_02205_b200.binding as B
lib = B.load_library()
f = lib["_ZN3psb12launch_routeEPKvPKfPKhRK14psb_route_descPiPfS9_S9_S9_PvP11CUstream_st"]
f.restype, f.argtypes = C.c_int, [C.c_void_p] * 11
d = B.psb_route_desc(B.PSB_DT_F32, 0, {tokens}, {experts}, 4, 1, 1, 1, 1, 1.0, {experts})
P, before = 1 << 20, lib.psb_launch_count()
assert f(P, None, None, C.addressof(d), P, P, P, P, P, P, None) != 0
assert lib.psb_launch_count() - before <= 1, lib.psb_launch_count() - before
"""


@pytest.mark.parametrize("tokens,experts", [(64, 64), (1000, 64), (1000, 256), (50000, 512)])
def test_routing_stops_at_a_failed_launch(tokens, experts):
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="")
    r = subprocess.run([sys.executable, "-c", _ROUTE.format(tokens=tokens, experts=experts)], cwd=ROOT, env=env, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-1500:]
