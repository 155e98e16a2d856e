"""Prefix trees of drafts and acceptance of their paths on the GPU, bit for bit against the
plain oracle: random drafts over few tokens (many shared prefixes), budgets that cut a draft,
drafts that cannot be accepted, one-token drafts, words that end inside a mask row."""
import numpy as np
import pytest
import torch

from oracle import verify as ov

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print(*a, flush=True)


def up(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).to(DEV)


def drafts_of(rng, B, r, length, vocab, eos):
    d = rng.integers(0, vocab, (B, r, length)).astype(np.int32)
    d[:, :, 0] = np.where(rng.random((B, r)) < 0.9, 5, 6)
    return d, rng.integers(-1, r + 2, B).astype(np.int32), np.full(B, 5, np.int32)


CASES = [  # B, r, length, vocab, N, eos
    (1, 1, 1, 3, 1, 0), (3, 1, 9, 3, 9, 0), (5, 10, 10, 3, 91, 0), (4, 10, 10, 2, 30, 1),
    (2, 100, 20, 3, 1000, 0), (3, 64, 6, 3, 64, 0), (3, 64, 6, 3, 65, 0), (2, 7, 40, 2, 128, -3),
    (2, 1024, 5, 6, 1024, 0), (1, 1024, 30, 3, 700, 2), (2, 3, 4096, 2, 1024, 7),
    (300, 3, 20, 2, 58, 0)]


@pytest.mark.parametrize("B,r,length,vocab,N,eos", CASES, ids=str)
def test_tree(gpu_lib, B, r, length, vocab, N, eos):
    from paper_2502_15572_amd import draft_tree
    say("tree", B, r, length, vocab, N, eos)
    rng = np.random.default_rng(B * 1000 + r + N)
    d, count, first = drafts_of(rng, B, r, length, vocab, eos)
    if length > 1000:          # two long drafts that part late, and one inside the other
        d[:, :] = d[:, :1]
        d[:, :, 0] = 5
        d[:, 1, 900:] ^= 1
        d[:, 2, 1020:] = eos
    want = ov.draft_tree(d, count, first, N, eos)
    tok, par, dep, mask, nodes = draft_tree(up(d), up(count), up(first), N, eos)
    assert np.array_equal(nodes.cpu().numpy(), want[4])
    assert np.array_equal(tok.cpu().numpy(), want[0])
    assert np.array_equal(par.cpu().numpy(), want[1])
    assert np.array_equal(dep.cpu().numpy(), want[2])
    assert np.array_equal(mask.cpu().numpy().view(np.uint64), ov.mask_words(want[3], N))


def test_tree_default_budget_out_and_empty_batch(gpu_lib):
    from paper_2502_15572_amd import draft_tree
    say("tree: defaults")
    rng = np.random.default_rng(1)
    d, count, first = drafts_of(rng, 3, 6, 5, 4, 0)
    a = draft_tree(up(d), up(count), up(first))
    assert a[0].shape == (3, 25)
    out = tuple(torch.full_like(t, -7) for t in a)
    b = draft_tree(up(d), up(count), up(first), out=out)
    assert all(x is y for x, y in zip(b, out)) and all(torch.equal(x, y) for x, y in zip(a, b))
    e = draft_tree(up(d[:0]), up(count[:0]), up(first[:0]))
    assert e[3].shape == (0, 25, 1)


def tree_of(rng, B, N):
    """Random trees: parents before children, few tokens, siblings that share a token."""
    token = rng.integers(0, 6, (B, N)).astype(np.int32)
    parent = np.array([[-1] + [int(rng.integers(max(0, u - 4), u)) for u in range(1, N)]
                       for _ in range(B)], np.int32)
    return token, parent, rng.integers(-1, N + 2, B).astype(np.int32)


ACCEPT = [  # B, N, V, most, dtype, pad
    (1, 1, 1, 1, "f32", 0), (4, 30, 6, 30, "f32", 0), (5, 64, 7, 10, "bf16", 3),
    (3, 91, 1000, 91, "f16", 0), (2, 20, 32000, 8, "f32", 0), (2, 17, 50257, 17, "bf16", 0),
    (70, 12, 4099, 3, "f16", 5), (1, 1024, 333, 1024, "bf16", 1), (9, 8, 128001, 8, "bf16", 7)]


@pytest.mark.parametrize("B,N,V,most,dtype,pad", ACCEPT, ids=str)
def test_accept(gpu_lib, B, N, V, most, dtype, pad):
    """Logits of few levels (ties everywhere), the winners among the tree's tokens."""
    from paper_2502_15572_amd import accept_drafts
    say("accept", B, N, V, most, dtype, pad)
    rng = np.random.default_rng(V + N)
    token, parent, nodes = tree_of(rng, B, N)
    x = rng.integers(-3, 1, (B, N, V)).astype(np.float32)
    b, u = np.indices((B, N))
    x[b, u, rng.integers(0, min(6, V), (B, N))] = 1.0
    x[rng.random((B, N, V)) < 0.01] = -np.inf
    x[rng.random((B, N, V)) < 0.01] = np.nan
    x[rng.random((B, N)) < 0.02] = np.nan
    want = ov.accept(x.astype(np.float64), token, parent, nodes, most)
    buf = torch.full((B, N, V + pad), 99.0, dtype={"f32": torch.float32, "f16": torch.float16,
                                                  "bf16": torch.bfloat16}[dtype], device=DEV)
    buf[:, :, :V] = torch.from_numpy(x).to(DEV)
    got = accept_drafts(buf[:, :, :V], up(token), up(parent), up(nodes), most)
    for w, g in zip(want, got):
        assert np.array_equal(w, g.cpu().numpy())


def test_accept_unaligned_rows_and_last_token(gpu_lib):
    """Rows that start at every offset within 16 bytes; the winner first, last, and everywhere."""
    from paper_2502_15572_amd import accept_drafts
    say("accept: offsets")
    token, parent, nodes = up([[3, 1]]), up([[-1, 0]]), up([1])
    for dtype in (torch.float32, torch.bfloat16):
        for V in (1, 5, 1023, 4096):
            buf = torch.zeros(2 * V + 64, dtype=dtype, device=DEV)
            for off in range(9):
                x = buf[off:off + 2 * V].view(1, 2, V)
                for w in sorted({0, V - 1, V // 2}):
                    buf.fill_(50.0)
                    x.zero_()
                    x[0, 0, w] = 1.0
                    assert accept_drafts(x, token, parent, nodes)[2].item() == w, (V, off, w)
                x.fill_(-float("inf"))
                assert accept_drafts(x, token, parent, nodes)[2].item() == 0


def test_accept_zeros_of_both_signs_and_infinities(gpu_lib):
    """-0 and +0 tie, +inf is the largest, the first of them wins."""
    from paper_2502_15572_amd import accept_drafts
    say("accept: zeros")
    inf = float("inf")
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        x = torch.full((1, 4, 3000), -1.0, dtype=dtype, device=DEV)
        x[0, 0, 7], x[0, 0, 2900] = -0.0, 0.0              # -> 7
        x[0, 1, 1], x[0, 1, 2] = 0.0, -0.0                 # -> 1
        x[0, 2, 2048], x[0, 2, 2999], x[0, 2, 5] = inf, inf, 60000.0   # -> 2048
        x[0, 3] = -inf
        x[0, 3, :9] = float("nan")                         # -> 9
        path, n, nxt = accept_drafts(x, up([[0, 7, 1, 2048]]), up([[-1, 0, 1, 2]]), up([4]))
        assert path.tolist() == [[0, 1, 2, 3]] and n.tolist() == [4] and nxt.tolist() == [9]


@pytest.mark.parametrize("bits,dtype", [(0x7f81, torch.bfloat16), (0xff81, torch.bfloat16),
                                        (0x7f800001, torch.float32), (0x7d01, torch.float16),
                                        (0x7fc00000, torch.float32), (0xffff, torch.float16)])
def test_accept_among_nans(gpu_lib, bits, dtype):
    """Quiet and signalling NaNs, of either sign, at every place beside the largest logit."""
    from paper_2502_15572_amd import accept_drafts
    say("accept: NaN", hex(bits), dtype)
    V, size = 4099, torch.finfo(dtype).bits // 8
    raw = {2: torch.int16, 4: torch.int32}[size]
    nan = torch.tensor([bits], dtype=torch.int64).to(raw).item() if bits < 1 << (8 * size - 1) \
        else bits - (1 << 8 * size)
    for hole in range(8):                                  # what is not NaN in every 8 elements
        for sign in (1.0, -1.0):
            x = torch.full((1, 2, V), nan, dtype=raw, device=DEV).view(dtype)
            x[:, :, hole::8] = -2.0
            x[0, 0, 2048 + hole] = sign
            x[0, 1, 4088 + hole] = sign * 0.5
            path, n, nxt = accept_drafts(x, up([[0, 2048 + hole]]), up([[-1, 0]]), up([2]))
            assert path.tolist() == [[0, 1]] and nxt.tolist() == [4088 + hole]
