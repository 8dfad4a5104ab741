"""Host threads that make their first calls of the paged operators at the same time, each on a stream of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import threading
import torch
import paper_2512_14481_b200 as P

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
work = []
for n in range(8):
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.zeros((4, 64, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = torch.randn((3, 50, 2, 64), generator=g, device="cuda").to(torch.bfloat16)
    cache = P.KVCache(k, v)
    batch = P.PagedBatch(i32([[0, 1, 2, 3]]), i32([50]), i32([0, 50]), 50, 50, 50)
    ws = torch.empty(P.sasq_paged_attention_workspace(cache, batch, 2), dtype=torch.uint8, device="cuda")
    work.append((cache, batch, x, torch.empty_like(x[0]), ws, torch.cuda.Stream()))
torch.cuda.synchronize()
gate, errors = threading.Barrier(8), []

def go(cache, batch, x, out, ws, stream):
    try:
        gate.wait(60)
        for _ in range(20):
            P.sasq_rope_kv_append(cache, batch, None, x[1], x[2], None, None, stream=stream)
            P.sasq_paged_attention(cache, batch, x[0], out, ws, stream=stream)
    except Exception as e:
        errors.append(e)

threads = [threading.Thread(target=go, args=w) for w in work]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert not errors, errors
assert P.sasq_device_status() == 0
for cache, batch, x, out, ws, _ in work:
    q, k, v = x.double().transpose(1, 2)
    s = (q @ k.transpose(1, 2) / 8).masked_fill(torch.ones(50, 50, device="cuda").triu(1).bool(), -torch.inf)
    p = torch.softmax(s, -1)
    # u |out| + A (u + small), A = sum p |v|, u = 2^-8: probabilities and outputs are rounded to bf16
    tol = 2.0 ** -8 * (p @ v).abs() + (p @ v.abs()) * (2.0 ** -8 + 2.0 ** -12)
    assert ((out.double().transpose(0, 1) - p @ v).abs() <= tol).all()
print("fine")
"""


def test_first_calls_from_many_threads():
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "fine" in run.stdout, run.stdout + run.stderr
