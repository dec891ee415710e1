"""A call reports its own launches, not what an earlier call has left behind."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Launches on a stream whose capture is no longer valid are refused by the runtime on the host.  (In a process of its own: the capture cannot
# be ended properly.)
_SCRIPT = """
import torch
import paper_1904_02205_b200 as psb
ctx = psb.Context(0)
x = torch.randn(40, 256, device="cuda")
a, sa = ctx.quantize_fp8(x)
b, sb = ctx.quantize_fp8(torch.randn(128, 256, device="cuda"), block_rows=128)
weights, slot = torch.ones(40, 2, device="cuda"), torch.zeros(40, 2, dtype=torch.int32, device="cuda")
offsets = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
y = torch.empty(40, 128, dtype=torch.bfloat16, device="cuda")
z = torch.empty(40, 256, device="cuda")
calls = dict(gemm_fp8=lambda s=None: ctx.gemm_fp8(a, sa, b, sb, out=y, stream=s),
             gemm_fp8_experts=lambda s=None: ctx.gemm_fp8_experts(a, sa, b[None], sb[None], offsets, out=y, stream=s),
             quantize_fp8=lambda s=None: ctx.quantize_fp8(x, out=(a, sa), stream=s),
             combine_experts=lambda s=None: ctx.combine_experts(x, weights, slot, out=z, stream=s))
for f in calls.values():
    f()
torch.cuda.synchronize()
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.stream(side):
    graph.capture_begin()
    try:
        torch.cuda.synchronize()
    except RuntimeError:
        pass
    failed = []
    for name, f in calls.items():
        for after in calls:
            try:
                f(side)
            except psb.PsbError as e:
                failed.append(name)
                assert e.status == psb.PSB_ERR_CUDA
            calls[after](torch.cuda.default_stream())
    assert len(failed) == len(calls) ** 2, failed
    try:
        graph.capture_end()
    except RuntimeError:
        pass
print("FINE", flush=True)
import os
os._exit(0)
"""


def test_a_launch_that_fails_is_not_reported_by_the_next_call():
    r = subprocess.run([sys.executable, "-c", _SCRIPT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert "FINE" in r.stdout, r.stderr[-2000:]
