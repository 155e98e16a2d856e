"""Attention over 8-bit values far apart in size, seen with weights that bring them together again:
the outputs are ordinary numbers, whatever the exponents of the rows."""
import numpy as np
import pytest
import torch

from oracle import verify as ov
from test_gpu_attend import Case, say

pytestmark = pytest.mark.gpu


def put(c, name, p, row):
    """A row of every head at position p of sequence 0."""
    codes, exp = ov.quantise(row)
    at = c.table[0, p // c.page], slice(None), p % c.page
    c.bits[name][at], c.exp[name][at], c.val[name][at] = codes, exp, ov.dequantise(codes, exp)
    return int(exp[0]) - 127


# score of the large values, exponent of their rows: e^score 2^(exponent + 8) is 2^5 to 2^12
LARGE = [(-16.0, 27), (-32.0, 46), (-48.0, 68), (-56.0, 80), (-16.0, 20), (-4.0, 0)]


@pytest.mark.parametrize("n,dim", [(1, 128), (1, 256), (9, 64), (20, 128), (90, 64), (150, 128),
                                   (70, 256)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_large_values_with_small_weights(gpu_lib, n, dim, dtype):
    from paper_2502_15572_amd import paged_attention
    for score, e in LARGE:
        say("attend: values of 2^%d" % (e + 8), n, dim, dtype)
        c = Case(n + dim, [200], [n], 2, 2, dim, 16, dtype, "f8")
        rng = np.random.default_rng(e)
        c.q.zero_()
        c.q[..., 0] = 1.0                    # a key's score is its first element
        for p in (3, 40, 41, 150):
            key = np.zeros((2, dim))
            key[:, 0] = score
            put(c, "k", p, key)
            row = rng.uniform(-1, 1, (2, dim)) * 2.0 ** (e + 8)
            row[:, 5], row[:, 1::4] = 1.5 * 2.0 ** (e + 8), 0.0
            assert put(c, "v", p, row) == e
        args, kw = c.tensors()
        out, lse = paged_attention(*args, **kw, scale=1.0, with_lse=True)
        out = out.view(n, c.H, dim).to(torch.float64).cpu().numpy()
        lse = lse.view(n, c.H).to(torch.float64).cpu().numpy()
        L = 200 + n
        at = np.arange(L)
        k, v, ve = (t[c.table[0, at // 16], :, at % 16] for t in (
            c.val["k"], c.val["v"], c.exp["v"].astype(np.int64) - 127))
        want, wl, mag, size = ov.attend(c.q.to(torch.float64).numpy(), k, v, c.see(0), 1.0)
        # test_gpu_attend's tolerance; and f16 weights, times their value's power of two, are below
        # their normal numbers off by 2^-35 of the row's largest, each against a code of at most 448
        u = torch.finfo(c.q.dtype).eps / 2
        ds = (dim + 4) * 2.0 ** -24 * size
        rel = 2.2 * ds + 2.0 ** -20 + (2 * L + 64) * 2.0 ** -24
        tol = u * np.abs(want) + (u + rel)[..., None] * mag + 1e-38
        if dtype == "f16":
            w = np.exp(k[:, 0, 0][None] - wl[:, :1]) * c.see(0)
            w2 = np.exp(k[:, 1, 0][None] - wl[:, 2:3]) * c.see(0)
            top = np.stack([(w * 2.0 ** ve[:, 0]).max(1), (w2 * 2.0 ** ve[:, 1]).max(1)], 1)
            tol = tol + 2.0 ** -25 + (L * 448 * 2.0 ** -35 * np.repeat(top, 2, 1))[..., None]
        assert np.isfinite(out).all()
        err = np.abs(out - want)
        say("worst error / tolerance %.3f, largest output %.0f" % ((err / tol).max(),
                                                                   np.abs(want).max()))
        assert (err <= tol).all()
        assert (np.abs(lse - wl) <= ds + 2.0 ** -20 + (L + 8) * 2.0 ** -24
                + 2.0 ** -22 * np.abs(wl)).all()


@pytest.mark.parametrize("length", [5, 0, -3, -(1 << 31)])
def test_a_chunk_of_2_to_the_30_rows(gpu_lib, length):
    """Of far fewer tokens than rows: the rows before the first position see nothing."""
    from paper_2502_15572_amd import paged_attention
    say("attend: 2^30 rows, length", length)
    dev, n = "cuda:0", (1 << 30) + 200
    x = torch.randn(3, 8, generator=torch.Generator().manual_seed(1)).to(torch.float16)
    pages = torch.stack([x[0], x[1]]).view(2, 1, 1, 1, 8).expand(2, 1, 1, 16, 8).contiguous().to(dev)
    q = x[2].to(dev).expand(1, n, 1, 8)
    table = torch.zeros(1, 1, dtype=torch.int32, device=dev)
    lengths = torch.tensor([length], dtype=torch.int32, device=dev)
    out = torch.empty(1, n, 1, 8, dtype=torch.float16, device=dev)
    out[0, -400:] = 7.0
    paged_attention(q, pages[0], pages[1], table, lengths, out=out)
    sees = max(0, length)                    # every key and value alike: the output is the value
    last = out[0, -400:, 0].cpu()
    assert (last[:400 - sees] == 0).all()
    assert (last[400 - sees:] - x[1]).abs().le(2.0 ** -10 * x[1].abs()).all()


@pytest.mark.parametrize("dtype,cache", [("f16", "f8"), ("bf16", "f8"), ("f16", "f16")])
@pytest.mark.parametrize("n,ctx", [(1, 1), (7, 1), (1, 900), (40, 3), (130, 70)])
def test_logarithms_of_sums_near_the_reference(gpu_lib, n, ctx, dtype, cache):
    """Scores of zero: a row's sum is the number of its positions, times a power of two that comes
    from its values' size.  The weights and their sum are exact, the logarithm is off by two steps of
    its fraction, of the sum with the exponent and of the product with ln 2."""
    from paper_2502_15572_amd import paged_attention
    say("attend: logarithms", n, ctx, dtype, cache)
    for size in (0, 40, -40):
        c = Case(n, [ctx], [n], 2, 3, 72, 16, dtype, cache)
        if cache == "f8":
            c.exp["v"] = np.where(c.exp["v"] == 255, 255, c.exp["v"].astype(np.int64)
                                  + size).astype(np.uint8)
        args, kw = c.tensors()
        _, lse = paged_attention(*args, **kw, scale=0.0, with_lse=True)
        want = np.log(ctx + 1.0 + np.arange(n))[:, None]
        err = np.abs(lse.view(n, c.H).to(torch.float64).cpu().numpy() - want)
        say("worst %.2e" % err.max())
        assert (err <= 2.0 ** -22 * (1 + want)).all()
