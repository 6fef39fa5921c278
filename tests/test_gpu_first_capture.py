"""Grouped products and orthogonalised updates whose kernels run for the first time inside a stream capture, in a process of its own: after any first call of
the library on the device, every other first call may be a captured one."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import torch
import paper_2609_09095_b200 as oz

oz.oz_query_status()
gen = torch.Generator("cuda").manual_seed(1)
x = torch.randn(600, 264, device="cuda", generator=gen).bfloat16()
dy = torch.randn(600, 136, device="cuda", generator=gen).bfloat16()
w = torch.randn(3, 136, 264, device="cuda", generator=gen).bfloat16()
g = [torch.randn(2, 300, 260, device="cuda", generator=gen), torch.randn(2, 60, 500, device="cuda", generator=gen).bfloat16()]
offsets = torch.tensor([0, 100, 100, 600], device="cuda")
space = [torch.empty(oz.oz_orthogonalise_workspace_bytes(a.shape[2], a.shape[1], 2), dtype=torch.uint8, device="cuda") for a in g]


def calls(y, dw, o):
    oz.check(oz.oz_gemm_grouped(1, 136, 600, 264, 3, offsets, oz.OZ_BF16, w, 264, 136 * 264, x, 264, oz.OZ_F32, 0.0, y, 136))
    oz.check(oz.oz_gemm_grouped_wgrad(264, 136, 600, 3, offsets, oz.OZ_BF16, x, 264, dy, 136, oz.OZ_BF16, 0.0, dw, 264, 136 * 264))
    for a, s, r in zip(g, space, o):
        t = oz.OZ_F32 if a.dtype == torch.float32 else oz.OZ_BF16
        rows, cols = a.shape[1:]
        oz.check(oz.oz_orthogonalise(cols, rows, 2, t, a, cols, rows * cols, 5, (3.4445, -4.775, 2.0315), 1e-7, t, r, cols, rows * cols, s))


def results():
    return torch.zeros(600, 136, device="cuda"), torch.zeros(3, 136, 264, dtype=torch.bfloat16, device="cuda"), [torch.zeros_like(a) for a in g]


captured, eager = results(), results()
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
side.wait_stream(torch.cuda.current_stream())
with torch.cuda.graph(graph, stream=side):
    calls(*captured)
for _ in range(2):
    graph.replay()
torch.cuda.synchronize()
calls(*eager)
torch.cuda.synchronize()
assert oz.oz_query_status() in (oz.OZ_OK, oz.OZ_ERR_RANGE)
for a, b in zip([*captured[:2], *captured[2]], [*eager[:2], *eager[2]]):
    assert a.any() and torch.equal(a, b)
print("same")
"""


def test_kernels_run_first_in_a_capture():
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("same"), run.stderr[-2000:]
