"""Acceptance over rows of a few logits, which lie across 16-byte borders in every way: with and
without whole 16 bytes, row by row, the last of them at the end of the memory."""
import numpy as np
import pytest
import torch

from oracle import verify as ov
from test_gpu_tree import DEV, say, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=str)
def test_short_rows(gpu_lib, dtype):
    from paper_2502_15572_amd import accept_drafts
    rng = np.random.default_rng(0)
    B, N = 3, 7
    for V in list(range(1, 27)) + [31, 33]:
        for pad in (0, 1, 3):
            say("accept: rows of", V, pad, dtype)
            # a path through all nodes, each the lowest child of the one before, some left early
            token = rng.integers(0, V, (B, N)).astype(np.int32)
            parent = np.tile(np.arange(-1, N - 1, dtype=np.int32), (B, 1))
            x = rng.integers(-3, 1, (B, N, V)).astype(np.float32)
            for b in range(B):
                for u in range(N - 1 - 2 * b):
                    x[b, u, token[b, u + 1]] = 1.0
            nodes = np.full(B, N, np.int32)
            want = ov.accept(x.astype(np.float64), token, parent, nodes, N)
            flat = torch.full((B * N * (V + pad) - pad,), 9.0, dtype=dtype, device=DEV)
            rows = flat.as_strided((B, N, V), (N * (V + pad), V + pad, 1))
            rows.copy_(torch.from_numpy(x))
            got = accept_drafts(rows, up(token), up(parent), up(nodes))
            for w, g in zip(want, got):
                assert np.array_equal(w, g.cpu().numpy()), (V, pad)
