"""The operators of batch verification refuse what they cannot serve, before any device
work (CPU only)."""
import ctypes

import pytest
import torch

import paper_2502_15572_amd as dresd
from paper_2502_15572_amd import _lib

E = _lib.EINVAL
FAKE = 256                     # never dereferenced: arguments are checked first


def cache(k=FAKE, v=FAKE, ke=None, ve=None, pages=4, page=16, heads=2, dim=64, dtype=_lib.F16):
    return _lib.KvCache(k, v, ke, ve, pages, page, heads, dim, dtype)


BAD_CACHES = [dict(pages=0), dict(pages=1 << 31), dict(page=0), dict(page=12), dict(page=1 << 17),
              dict(heads=0), dict(heads=65536), dict(dim=0), dict(dim=4), dict(dim=68),
              dict(dim=264), dict(dtype=_lib.F32), dict(dtype=4)]
BAD_MEMORY = [dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2),
              dict(dtype=_lib.F8), dict(dtype=_lib.F8, ke=FAKE)]


def write(lib, c, k=FAKE, k_row=128, k_head=64, v=FAKE, v_row=128, v_head=64, dtype=_lib.F16,
          slots=FAKE, n=3):
    return lib.dresd_kv_write(c, k, k_row, k_head, v, v_row, v_head, dtype, slots, n, None)


def read(lib, c, slots=FAKE, n=3, dtype=_lib.F16, k=FAKE, v=FAKE):
    return lib.dresd_kv_read(c, slots, n, dtype, k, v, None)


def attend(lib, c, q=FAKE, q_row=256, q_head=64, dtype=_lib.F16, q_heads=4, starts=None, n=2, B=3,
           T=6, table=FAKE, width=5, lengths=FAKE, mask=None, words=0, scale=0.1, out=FAKE):
    return lib.dresd_paged_attention(c, q, q_row, q_head, dtype, q_heads, starts, n, B, T, table,
                                     width, lengths, mask, words, scale, out, None, None, 0, None)


@pytest.mark.parametrize("bad", BAD_CACHES + BAD_MEMORY, ids=str)
def test_bad_caches(bad):
    lib = _lib.load()
    for call in (write, read, attend):
        assert call(lib, cache(**bad)) == E
        assert lib.dresd_last_error()
    if bad in BAD_MEMORY:      # no tokens: nothing is touched
        assert write(lib, cache(**bad), n=0) == read(lib, cache(**bad), n=0) == 0
        assert attend(lib, cache(**bad), T=0, B=0) == 0


def test_no_cache():
    lib = _lib.load()
    for call in (write, read, attend):
        assert call(lib, None) == E
    need = ctypes.c_int64()
    assert lib.dresd_paged_attention_workspace(None, 4, 0, 2, 3, 6, 5, ctypes.byref(need)) == E
    assert lib.dresd_paged_attention_workspace(cache(), 4, 0, 2, 3, 6, 5, None) == E


def test_bad_tokens():
    lib = _lib.load()
    for kw in [dict(k=None), dict(v=None), dict(slots=None), dict(dtype=_lib.F8), dict(dtype=-1),
               dict(n=-1), dict(n=1 << 30), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(k_row=132),
               dict(v_head=4), dict(k_row=-128), dict(v_row=1 << 41)]:
        assert write(lib, cache(), **kw) == E, kw
    for kw in [dict(k=None), dict(v=None), dict(slots=None), dict(dtype=_lib.F8), dict(n=-1),
               dict(n=1 << 30), dict(k=FAKE + 4), dict(v=FAKE + 8)]:
        assert read(lib, cache(), **kw) == E, kw


def test_bad_attention():
    lib = _lib.load()
    for kw in [dict(q=None), dict(table=None), dict(lengths=None), dict(out=None),
               dict(dtype=_lib.F32), dict(dtype=_lib.BF16), dict(dtype=_lib.F8), dict(q_heads=0),
               dict(q_heads=3), dict(q_heads=-2), dict(B=-1), dict(T=5), dict(n=-2), dict(T=-1),
               dict(width=0), dict(mask=FAKE, words=0), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(q=FAKE + 4), dict(out=FAKE + 8), dict(q_row=260),
               dict(q_head=-64), dict(n=1 << 29, B=2, T=1 << 30)]:
        assert attend(lib, cache(), **kw) == E, kw
    need = ctypes.c_int64()
    assert lib.dresd_paged_attention_workspace(cache(), 3, 0, 2, 3, 6, 5, ctypes.byref(need)) == E
    assert lib.dresd_paged_attention_workspace(cache(), 4, 0, 2, 3, 7, 5, ctypes.byref(need)) == E


def test_bad_trees():
    lib = _lib.load()
    F = FAKE

    def tree(drafts=F, count=F, first=F, B=1, r=4, length=4, N=13, token=F, parent=F, depth=F,
             mask=F, nodes=F):
        return lib.dresd_draft_tree(drafts, count, first, B, r, length, 0, N, token, parent, depth,
                                    mask, nodes, None)

    for kw in [dict(drafts=None), dict(count=None), dict(first=None), dict(B=-1), dict(r=0),
               dict(r=1025), dict(length=0), dict(length=4097), dict(N=0), dict(N=1025),
               dict(token=None), dict(parent=None), dict(depth=None), dict(mask=None),
               dict(nodes=None)]:
        assert tree(**kw) == E, kw
    assert tree(B=0, drafts=None) == 0


def test_bad_acceptance():
    lib = _lib.load()
    F = FAKE

    def accept(logits=F, dtype=0, row=100, V=100, token=F, parent=F, nodes=F, B=1, N=4, most=4,
               path=F, accepted=F, nxt=F):
        return lib.dresd_accept_drafts(logits, dtype, row, V, token, parent, nodes, B, N, most,
                                       path, accepted, nxt, None)

    for kw in [dict(logits=None), dict(token=None), dict(parent=None), dict(nodes=None),
               dict(path=None), dict(accepted=None), dict(nxt=None), dict(dtype=3), dict(row=99),
               dict(V=0), dict(V=(1 << 30) + 1, row=1 << 31), dict(B=-1), dict(N=0), dict(N=1025),
               dict(most=0), dict(most=1025), dict(logits=F + 2)]:
        assert accept(**kw) == E, kw
    assert accept(B=0, logits=None) == 0


def test_python_refuses_cpu_tensors_and_wrong_shapes():
    i32 = torch.int32
    d, c, f = torch.zeros(2, 3, 4, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(2, dtype=i32)
    with pytest.raises(TypeError, match="GPU"):
        dresd.draft_tree(d, c, f)
    for args, err in [((d.long(), c, f), TypeError), ((d, c[:1], f), ValueError),
                      ((d.transpose(1, 2), c, f), ValueError), ((d, c, f, 2000), ValueError)]:
        with pytest.raises(err):
            dresd.draft_tree(*args)
    kp = torch.zeros(3, 2, 16, 64, dtype=torch.float16)
    k = torch.zeros(5, 2, 64, dtype=torch.float16)
    s = torch.zeros(5, dtype=torch.int64)
    f8 = kp.to(torch.float8_e4m3fn)
    e = torch.zeros(3, 2, 16, dtype=torch.uint8)
    with pytest.raises(TypeError, match="GPU"):
        dresd.kv_write(k, k, s, kp, kp)
    with pytest.raises(TypeError, match="GPU"):
        dresd.kv_read(s, kp, kp)
    for args, err in [((k, k.float(), s, kp, kp), ValueError), ((k, k, s.int(), kp, kp), TypeError),
                      ((k, k, s[:4], kp, kp), ValueError), ((k[..., :32], k[..., :32], s, kp, kp),
                                                            ValueError),
                      ((k, k, s, kp.float(), kp.float()), TypeError),
                      ((k, k, s, kp, kp[:2]), ValueError), ((k, k, s, f8, f8), ValueError),
                      ((k, k, s, kp, kp, e, e), ValueError), ((k, k, s, f8, f8, e, None),
                                                              ValueError),
                      ((k, k, s, f8, f8, e, e[:2]), ValueError),
                      ((k, k, s, kp.transpose(1, 2), kp), ValueError)]:
        with pytest.raises(err):
            dresd.kv_write(*args)
    q = torch.zeros(2, 3, 4, 64, dtype=torch.float16)
    t, n = torch.zeros(2, 1, dtype=i32), torch.zeros(2, dtype=i32)
    with pytest.raises(TypeError, match="GPU"):
        dresd.paged_attention(q, kp, kp, t, n)
    m = torch.zeros(2, 3, 1, dtype=torch.int64)
    for args, kw, err in [((q.float(), kp, kp, t, n), {}, TypeError),
                          ((q[:1], kp, kp, t, n), {}, ValueError),
                          ((q, kp, kp, t[:1], n), {}, ValueError),
                          ((q, kp, kp, t, n.long()), {}, TypeError),
                          ((q[..., :32], kp, kp, t, n), {}, ValueError),
                          ((q, kp, kp, t, n), dict(mask=m[:, :2]), ValueError),
                          ((q, kp, kp, t, n), dict(starts=n), ValueError),
                          ((q, kp, kp, t, n), dict(starts=torch.zeros(3, dtype=i32)), ValueError),
                          ((q[:, :, ::2, :], kp, kp, t, n), dict(out=(q, q), with_lse=False),
                           (TypeError, ValueError))]:
        with pytest.raises(err):
            dresd.paged_attention(*args, **kw)
    x = torch.zeros(2, 3, 10)
    tk = torch.zeros(2, 3, dtype=i32)
    with pytest.raises(TypeError, match="GPU"):
        dresd.accept_drafts(x, tk, tk, n)
    for args, err in [((x[0], tk, tk, n), ValueError), ((x, tk[:1], tk, n), ValueError),
                      ((x.transpose(1, 2), tk, tk, n), ValueError),
                      ((x, tk.long(), tk, n), TypeError), ((x, tk, tk, n[:1]), ValueError)]:
        with pytest.raises(err):
            dresd.accept_drafts(*args)


def test_rows_of_more_than_31_bits_of_bytes():
    """Offsets within a row of logits are 32 bits, past its end by what a workgroup reads at once."""
    lib = _lib.load()
    F, V = FAKE, (1 << 29) + 1
    assert lib.dresd_accept_drafts(F, 0, V, V, F, F, F, 1, 4, 4, F, F, F, None) == E


def test_more_than_a_launch_takes():
    """A launch has fewer than 2^32 threads: 1,024 a query in trees and acceptance, 8, 16 or 32 a
    row in cache writes and reads."""
    lib = _lib.load()
    F = FAKE
    for B in (1 << 22, (1 << 31) - 1):
        assert lib.dresd_draft_tree(F, F, F, B, 4, 4, 0, 13, F, F, F, F, F, None) == E
        assert lib.dresd_accept_drafts(F, 0, 100, 100, F, F, F, B, 4, 4, F, F, F, None) == E
    for dim, most in ((64, 1 << 29), (72, 1 << 28), (128, 1 << 28), (136, 1 << 27), (256, 1 << 27)):
        c = cache(dim=dim, heads=2)
        assert write(lib, c, k_row=2 * dim, k_head=dim, v_row=2 * dim, v_head=dim,
                     n=most // 2 - 15) == E
        assert read(lib, c, n=most // 2 - 15) == E
