"""Pins of the verification oracle by closed forms and by torch's own formats (CPU only)."""
import numpy as np
import pytest
import torch

from oracle import verify as ov


def test_tree_by_hand():
    #   7 - 1 - 2 - 3        drafts 0 and 1 share 7 1 2; draft 2 leaves after 7; draft 3 starts
    #    \    \- (2) - 4     with another token; draft 4 repeats draft 0; draft 5 ends at once
    d = np.array([[[7, 1, 2, 3], [7, 1, 2, 4], [7, 5, 0, 0], [8, 1, 2, 3], [7, 1, 2, 3],
                   [0, 0, 0, 0]]], np.int32)
    tok, par, dep, anc, n = ov.draft_tree(d, [6], [7], 8)
    assert n.tolist() == [6]
    assert tok[0].tolist() == [7, 1, 2, 3, 4, 5, 0, 0]
    assert par[0].tolist() == [-1, 0, 1, 2, 2, 0, -1, -1]
    assert dep[0].tolist() == [0, 1, 2, 3, 3, 1, 0, 0]
    assert anc[0] == [{0}, {0, 1}, {0, 1, 2}, {0, 1, 2, 3}, {0, 1, 2, 4}, {0, 5}]
    assert ov.draft_tree(d, [6], [7], 4)[4].tolist() == [4]
    assert ov.draft_tree(d, [0], [7], 4)[4].tolist() == [1]
    assert ov.mask_words(anc, 8)[0, :, 0].tolist() == [1, 3, 7, 15, 23, 33, 0, 0]


def test_e4m3_is_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(ov.e4m3_value(codes), want, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).uniform(-448, 448, 4000),
                        np.random.default_rng(1).uniform(-0.02, 0.02, 4000),
                        (ov.E4M3[1:] + ov.E4M3[:-1]) / 2, -(ov.E4M3[1:] + ov.E4M3[:-1]) / 2,
                        [0.0, 448.0, -448.0, np.nan]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = ov.e4m3(x)
    nan = np.isnan(x)
    assert np.array_equal(got[~nan], want[~nan]) and (got[nan] & 127 == 127).all()


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.5, 1), (1.75, -8), (1.76, -7), (1.0, -8),
                                   (0.0, -9), (1e-40, -126), (65504.0, 8)])
def test_exponent_is_the_smallest_that_holds_the_row(top, e):
    codes, exp = ov.quantise(np.array([[top, -top / 3, 0.0]]))
    assert int(exp[0]) - 127 == e
    assert np.abs(ov.e4m3_value(codes)).max() <= 448
    back = ov.dequantise(codes, exp)
    # stored again, the same values (by other codes where the largest was rounded down to 224)
    assert np.array_equal(ov.dequantise(*ov.quantise(back)), back)


def test_attention_closed_forms():
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((5, 1, 4)), rng.standard_normal((5, 1, 4))
    k[3], v[3] = np.nan, np.inf                       # not seen
    see = np.array([[1, 1, 1, 0, 0], [0, 0, 0, 0, 0], [0, 0, 0, 0, 1]], bool)
    out, lse, mag, _ = ov.attend(np.zeros((3, 2, 4)), k, v, see, 0.5)
    assert np.allclose(out[0, 1], v[:3, 0].mean(0)) and np.allclose(lse[0], np.log(3))
    assert (out[1] == 0).all() and (lse[1] == -np.inf).all()
    assert np.allclose(out[2, 0], v[4, 0]) and np.allclose(mag[2, 0], np.abs(v[4, 0]))


def test_acceptance_by_hand():
    tok = np.array([[7, 1, 2, 3, 4, 5]], np.int32)
    par = np.array([[-1, 0, 1, 2, 2, 0]], np.int32)
    x = np.full((1, 6, 9), -1.0)
    x[0, 0, 1] = x[0, 1, 2] = x[0, 2, 4] = x[0, 4, 8] = 1.0
    x[0, 4, 6] = 1.0                                   # tie: the lower token
    p, a, g = ov.accept(x, tok, par, [6], 6)
    assert p[0].tolist() == [0, 1, 2, 4, -1, -1] and a[0] == 4 and g[0] == 6
    p, a, g = ov.accept(x, tok, par, [3], 6)           # nodes 3 and up are not there
    assert a[0] == 3 and g[0] == 4
    p, a, g = ov.accept(x, tok, par, [6], 2)
    assert p[0].tolist() == [0, 1] and g[0] == 2
    assert ov.accept(x, tok, par, [0], 2)[1].tolist() == [0]
