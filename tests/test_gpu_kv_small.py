"""8-bit rows at the bottom of fp32: what is read back exactly, and in which type."""
import numpy as np
import pytest
import torch

from oracle import verify as ov
from test_gpu_kv import DEV, cached, new_cache, say

pytestmark = pytest.mark.gpu


def test_smallest_exponents_and_codes(gpu_lib):
    """Rows whose exponents are -126 to -122 and whose elements are the smallest codes: exact in
    fp32, and from -124 on in bf16 (before that the nearest number, ties to even)."""
    from paper_2502_15572_amd import kv_read, kv_write
    say("kv: smallest exponents")
    e = np.array([-126, -126, -125, -124, -123, -122])
    x = np.arange(64) * 2.0 ** -9 * np.where(np.arange(64) % 3, 1, -1)      # codes of 0 to 63 / 512
    x = np.broadcast_to(x, (6, 1, 64)).copy()
    x[1:, 0, 0] = 448.0                                    # (the first row has small codes alone)
    x *= 2.0 ** e[:, None, None]
    k = torch.from_numpy(x.astype(np.float32))
    kp, vp, ke, ve = new_cache("f8", 2, 1, 16, 64)
    s = torch.arange(6, device=DEV)
    kv_write(k.to(DEV), -k.to(DEV), s, kp, vp, ke, ve)
    bits, exp = ov.quantise(k.to(torch.float64).numpy())
    assert (exp[:, 0].astype(int) - 127 == e).all() and np.array_equal(cached(kp, s, 16), bits)
    want = torch.from_numpy(ov.dequantise(bits, exp))
    got, neg = kv_read(s, kp, vp, ke, ve, dtype=torch.float32)
    assert torch.equal(got.cpu().to(torch.float64), want) and torch.equal(got, -neg)
    kv_write(got, neg, s + 16, kp, vp, ke, ve)
    assert np.array_equal(cached(kp, s + 16, 16), bits)
    half = kv_read(s, kp, vp, ke, ve)[0]
    assert half.dtype == torch.bfloat16
    assert torch.equal(half.cpu().view(torch.int16),
                       want.to(torch.float32).to(torch.bfloat16).view(torch.int16))
    assert torch.equal(half.cpu().to(torch.float64)[3:], want[3:])
    kv_write(half, half, s + 16, kp, vp, ke, ve)
    assert np.array_equal(cached(kp, s + 16, 16)[3:], bits[3:])
