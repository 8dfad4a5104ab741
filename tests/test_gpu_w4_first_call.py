"""A process whose first call of the 4-bit operators is captured into a graph."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import torch
import paper_2512_14481_b200 as P
for T in (1, 5, 12, 20, 50):
    x = torch.randn((T, 1024), device="cuda").half()
    w = torch.randint(0, 256, (700, 512), device="cuda").to(torch.uint8)
    s = torch.rand((700, 8), device="cuda").half()
    y = torch.zeros((T, 700), device="cuda").half()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.sasq_w4_linear(x, w, s, y)
    assert not y.any()
    graph.replay()
    first = y.clone()
    P.sasq_w4_linear(x, w, s, y)
    assert torch.equal(first, y) and y.any(), T
cache = P.KVCache(*(torch.zeros((4, 16, 2, 32), dtype=torch.uint8, device="cuda") for _ in range(2)),
                  *(torch.ones((2, 64), device="cuda") for _ in range(2)))
i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
for n in (1, 40):
    batch = P.PagedBatch(i32([[3, 1, 0]]), i32([n]), i32([0, n]), n, n, 48)
    k, v = (2 * torch.randn((n, 2, 64), device="cuda").half() for _ in range(2))
    q, out = torch.randn((n, 8, 64), device="cuda").half(), torch.zeros((n, 8, 64), device="cuda").half()
    ws = torch.empty(max(16, P.sasq_paged_attention_workspace(cache, batch, 8)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.sasq_rope_kv_append(cache, batch, None, k, v, None, None)
        P.sasq_paged_attention(cache, batch, q, out, ws)
    graph.replay()
    first = out.clone()
    P.sasq_paged_attention(cache, batch, q, out, ws)
    assert torch.equal(first, out) and out.any(), n
assert P.sasq_device_status() == 0
print("done")
"""


def test_first_calls_are_captured():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "done" in done.stdout, done.stderr[-2000:]
