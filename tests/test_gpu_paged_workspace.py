"""The workspace of the paged attention: what the query says is enough for the call, whatever the shapes and host bounds."""
import random

import pytest
import torch

import paged_reference as R
import paper_2512_14481_b200 as P

pytestmark = pytest.mark.gpu


def test_a_workspace_of_the_queried_size_is_enough():
    """Random shapes and host bounds, the sequences themselves short: the call takes exactly what the query said, and
    writes nothing behind it."""
    rng = random.Random(4)
    guard = 4096
    for _ in range(150):
        group, K, D = rng.choice((1, 2, 4, 5, 8, 40)), rng.choice((1, 2, 8, 40)), rng.choice((64, 128))
        count, new = rng.choice((1, 2, 7, 30, 200)), rng.choice((0, 1, 2, 3, 9, 40, 300))
        if count * new * group * K > 8000:
            continue
        bt = R.Batch([rng.randint(0, 60) for _ in range(count)], [rng.randint(0, new) for _ in range(count)], group * K, K, D, 16,
                     rng.choice((torch.float16, torch.bfloat16)), rng.random() < 0.5, max_pages=4)
        cache, batch = bt.handles(P, rng.choice((None, 1, 17, 1000, 1 << 20)), rng.choice((None, 1, 200, 5000, 20000, 1 << 30)))
        n = P.sasq_paged_attention_workspace(cache, batch, bt.heads)
        ws = torch.full((n + guard,), 165, dtype=torch.uint8, device="cuda")
        out = torch.empty((bt.T, bt.heads, D), dtype=bt.dtype, device="cuda")
        P.sasq_paged_attention(cache, batch, bt.q, out, ws[:n])
        assert P.sasq_device_status() == 0
        assert (ws[n:] == 165).all()
        if n >= 16 and bt.T > 0:
            with pytest.raises(P.SasqError):
                P.sasq_paged_attention(cache, batch, bt.q, out, ws[:n - 1])
