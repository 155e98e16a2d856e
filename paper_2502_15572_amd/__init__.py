"""MI355X-native exact dense retrieval for DReSD (Dense Retrieval for
Speculative Decoding): a datastore of L2-normalised token embeddings mapped to
their next tokens (Section 3.5), searched by inner product (Eq. 3 with unit
norms) for the k best keys whose continuations become drafts (Section 3.6).

The search runs in hand-written gfx950 HIP kernels behind the C ABI of
``include/dresd.h``; this module only passes torch device pointers and the
current stream to it.
"""
from __future__ import annotations

import ctypes
import functools

from . import _lib
from ._lib import DresdError, K_MAX, NODES_MAX  # noqa: F401

__all__ = ["Index", "PartitionedIndex", "DresdError", "K_MAX", "transform", "pack_drafts",
           "draft_tree", "kv_write", "kv_read", "paged_attention", "accept_drafts", "NODES_MAX",
           "kmeans_assign", "kmeans_update", "kmeans_init", "train_partitions", "bw_probe",
           "release_cached"]

_DTYPES = None


def _dtype_code(t):
    import torch
    global _DTYPES
    if _DTYPES is None:
        _DTYPES = {torch.float32: _lib.F32, torch.float16: _lib.F16, torch.bfloat16: _lib.BF16}
    if t.dtype not in _DTYPES:
        raise TypeError("keys must be float32, float16 or bfloat16, not %s" % t.dtype)
    return _DTYPES[t.dtype]


def _stream_handle(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


# dresd_search_plan's scan kinds
SCAN_KINDS = {0: "single_tile", 1: "shared_key", 2: "single_tile_grouped", 3: "tiled",
              4: "whole_tile"}


class Index:
    """An exact inner-product index over ``keys[N, d]`` with values ``cont[N, L]``.

    Both tensors must be contiguous and on the current GPU; they are copied
    into library-owned memory, so they may be freed after construction.
    """

    def __init__(self, keys, cont, stream=None):
        import torch
        if not (keys.is_cuda and cont.is_cuda):
            raise ValueError("keys and continuations must be GPU tensors")
        if keys.dim() != 2 or cont.dim() != 2 or cont.shape[0] != keys.shape[0]:
            raise ValueError("keys must be [N, d] and continuations [N, L]")
        if cont.dtype != torch.int32:
            raise TypeError("continuations must be int32")
        keys = keys.contiguous()
        cont = cont.contiguous()
        self._lib = _lib.load()
        self._h = ctypes.c_void_p()
        self.N, self.d = int(keys.shape[0]), int(keys.shape[1])
        self.L = int(cont.shape[1])
        self.device = keys.device
        _lib.check(self._lib.dresd_index_create(
            ctypes.c_void_p(keys.data_ptr()), ctypes.c_void_p(cont.data_ptr()), self.N, self.d,
            self.L, _dtype_code(keys), _stream_handle(stream), ctypes.byref(self._h)))

    def search(self, queries, k: int, tokens: bool = True, out=None, stream=None, next_tok=None):
        """Top-k by inner product.  Returns ``(idx int64[B,k], score f32[B,k],
        tokens int32[B,k,L] or None)``.  With ``next_tok`` (int32 GPU tensor
        [B]) only rows whose continuation starts with the query's next token
        compete (Section 3.5); ranks past the matching rows hold idx -1,
        score -inf and zero tokens."""
        import torch
        if not queries.is_cuda or queries.dtype != torch.float32:
            raise TypeError("queries must be a float32 GPU tensor")
        if queries.dim() != 2 or queries.shape[1] != self.d:
            raise ValueError("queries must be [B, %d]" % self.d)
        q = queries.contiguous()
        B = int(q.shape[0])
        if next_tok is not None:
            if not next_tok.is_cuda or next_tok.dtype != torch.int32 or next_tok.numel() != B:
                raise TypeError("next_tok must be an int32 GPU tensor with one token per query")
            next_tok = next_tok.contiguous()
        if out is None:
            idx = torch.empty((B, k), dtype=torch.int64, device=q.device)
            score = torch.empty((B, k), dtype=torch.float32, device=q.device)
            tok = torch.empty((B, k, self.L), dtype=torch.int32, device=q.device) if tokens else None
        else:
            idx, score, tok = out
        tptr = ctypes.c_void_p(tok.data_ptr()) if tok is not None else None
        if next_tok is None:
            _lib.check(self._lib.dresd_search(
                self._h, ctypes.c_void_p(q.data_ptr()), B, int(k),
                ctypes.c_void_p(idx.data_ptr()), ctypes.c_void_p(score.data_ptr()), tptr,
                _stream_handle(stream)))
        else:
            _lib.check(self._lib.dresd_search_filtered(
                self._h, ctypes.c_void_p(q.data_ptr()), ctypes.c_void_p(next_tok.data_ptr()), B,
                int(k), ctypes.c_void_p(idx.data_ptr()), ctypes.c_void_p(score.data_ptr()), tptr,
                _stream_handle(stream)))
        return idx, score, tok

    def plan(self, B: int, k: int):
        sp, w, ws = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int64()
        kind, nl = ctypes.c_int32(), ctypes.c_int32()
        _lib.check(self._lib.dresd_search_plan(self._h, int(B), int(k), ctypes.byref(sp),
                                               ctypes.byref(w), ctypes.byref(ws),
                                               ctypes.byref(kind), ctypes.byref(nl)))
        return {"sample_passes": sp.value, "scan_waves": w.value, "workspace_bytes": ws.value,
                "scan_kernel": SCAN_KINDS[kind.value], "launches": nl.value}

    def profile(self, on: bool = True):
        _lib.check(self._lib.dresd_profile_enable(self._h, 1 if on else 0))

    def profile_read(self):
        a, b, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_int64()
        _lib.check(self._lib.dresd_profile_read(self._h, ctypes.byref(a), ctypes.byref(b),
                                                ctypes.byref(n)))
        return {"scan_ms": a.value, "search_ms": b.value, "searches": n.value}

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self._lib.dresd_index_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _search_out(B, k, L, tokens, device, out):
    import torch
    if out is not None:
        return out
    idx = torch.empty((B, k), dtype=torch.int64, device=device)
    score = torch.empty((B, k), dtype=torch.float32, device=device)
    tok = torch.empty((B, k, L), dtype=torch.int32, device=device) if tokens else None
    return idx, score, tok


class PartitionedIndex:
    """Partitioned (approximate) inner-product index: ``keys[N, d]`` with
    values ``cont[N, L]``, grouped into the partitions ``assign[N]`` (int32 in
    [0, P)) whose unit centroids are ``centroids[P, d]`` (float32).  A search
    probes the ``nprobe`` partitions with the best centroids and returns the
    exact top-k over their keys (the paper's approximate search, Section 3.5,
    read as an inverted file).  Everything is copied at construction."""

    def __init__(self, keys, cont, centroids, assign, stream=None):
        import torch
        for t in (keys, cont, centroids, assign):
            if not t.is_cuda:
                raise ValueError("all inputs must be GPU tensors")
        if keys.dim() != 2 or cont.dim() != 2 or cont.shape[0] != keys.shape[0]:
            raise ValueError("keys must be [N, d] and continuations [N, L]")
        if centroids.dtype != torch.float32 or centroids.dim() != 2 or \
                centroids.shape[1] != keys.shape[1]:
            raise TypeError("centroids must be float32 [P, d]")
        if cont.dtype != torch.int32 or assign.dtype != torch.int32 or \
                assign.numel() != keys.shape[0]:
            raise TypeError("continuations and assign must be int32; assign holds one id per key")
        keys, cont = keys.contiguous(), cont.contiguous()
        centroids, assign = centroids.contiguous(), assign.contiguous()
        self._lib = _lib.load()
        self._h = ctypes.c_void_p()
        self.N, self.d = int(keys.shape[0]), int(keys.shape[1])
        self.L = int(cont.shape[1])
        self.P = int(centroids.shape[0])
        _lib.check(self._lib.dresd_ivf_create(
            ctypes.c_void_p(keys.data_ptr()), ctypes.c_void_p(cont.data_ptr()), self.N, self.d,
            self.L, _dtype_code(keys), ctypes.c_void_p(centroids.data_ptr()), self.P,
            ctypes.c_void_p(assign.data_ptr()), _stream_handle(stream), ctypes.byref(self._h)))

    @classmethod
    def by_first_token(cls, keys, cont, stream=None):
        """Keys grouped by the first token of their continuation (one
        partition per distinct first token, in ascending token order, no
        centroids), for ``search_next_token``.  Copies everything."""
        import torch
        for t in (keys, cont):
            if not t.is_cuda:
                raise ValueError("all inputs must be GPU tensors")
        if keys.dim() != 2 or cont.dim() != 2 or cont.shape[0] != keys.shape[0]:
            raise ValueError("keys must be [N, d] and continuations [N, L]")
        if cont.dtype != torch.int32:
            raise TypeError("continuations must be int32")
        keys, cont = keys.contiguous(), cont.contiguous()
        self = cls.__new__(cls)
        self._lib = _lib.load()
        self._h = ctypes.c_void_p()
        self.N, self.d = int(keys.shape[0]), int(keys.shape[1])
        self.L = int(cont.shape[1])
        _lib.check(self._lib.dresd_ivf_create_by_token(
            ctypes.c_void_p(keys.data_ptr()), ctypes.c_void_p(cont.data_ptr()), self.N, self.d,
            self.L, _dtype_code(keys), _stream_handle(stream), ctypes.byref(self._h)))
        self.P = self.info()["P"]
        return self

    def search_next_token(self, queries, next_tok, k: int, tokens: bool = True, out=None,
                          stream=None):
        """Next-token-filtered exact top-k (the result of ``Index.search``
        with ``next_tok``) over an index from ``by_first_token``: each query
        scans only the keys whose continuation starts with its next token
        (``next_tok``, int32 GPU tensor [B])."""
        q = self._check_q(queries)
        B = int(q.shape[0])
        nt = self._next_tok(next_tok, B)
        if nt is None:
            raise TypeError("next_tok is required")
        idx, score, tok = _search_out(B, k, self.L, tokens, q.device, out)
        _lib.check(self._lib.dresd_ivf_search_next_token(
            self._h, ctypes.c_void_p(q.data_ptr()), ctypes.c_void_p(nt.data_ptr()), B, int(k),
            ctypes.c_void_p(idx.data_ptr()), ctypes.c_void_p(score.data_ptr()),
            ctypes.c_void_p(tok.data_ptr()) if tok is not None else None, _stream_handle(stream)))
        return idx, score, tok

    def _check_q(self, queries):
        import torch
        if not queries.is_cuda or queries.dtype != torch.float32:
            raise TypeError("queries must be a float32 GPU tensor")
        if queries.dim() != 2 or queries.shape[1] != self.d:
            raise ValueError("queries must be [B, %d]" % self.d)
        return queries.contiguous()

    @staticmethod
    def _next_tok(next_tok, B):
        import torch
        if next_tok is None:
            return None
        if not next_tok.is_cuda or next_tok.dtype != torch.int32 or next_tok.numel() != B:
            raise TypeError("next_tok must be an int32 GPU tensor with one token per query")
        return next_tok.contiguous()

    def search(self, queries, k: int, nprobe: int, tokens: bool = True, out=None, stream=None,
               next_tok=None):
        """Top-k over the keys of the ``nprobe`` best partitions (with
        ``next_tok``, int32 GPU tensor [B], only keys whose continuation starts
        with the query's next token).  Returns ``(idx, score, tokens)`` as
        ``Index.search``; ranks past the admitted keys hold idx -1, score -inf
        and zero tokens."""
        q = self._check_q(queries)
        B = int(q.shape[0])
        nt = self._next_tok(next_tok, B)
        idx, score, tok = _search_out(B, k, self.L, tokens, q.device, out)
        args = (ctypes.c_void_p(idx.data_ptr()), ctypes.c_void_p(score.data_ptr()),
                ctypes.c_void_p(tok.data_ptr()) if tok is not None else None,
                _stream_handle(stream))
        if nt is None:
            _lib.check(self._lib.dresd_ivf_search(
                self._h, ctypes.c_void_p(q.data_ptr()), B, int(k), int(nprobe), *args))
        else:
            _lib.check(self._lib.dresd_ivf_search_filtered(
                self._h, ctypes.c_void_p(q.data_ptr()), ctypes.c_void_p(nt.data_ptr()), B, int(k),
                int(nprobe), *args))
        return idx, score, tok

    def search_probes(self, queries, probes, k: int, tokens: bool = True, out=None, stream=None,
                      next_tok=None):
        """Top-k over the keys of the partitions in ``probes`` (int32 GPU
        tensor [B, S]; ids outside [0, P) ignored, repeats counted once),
        optionally next-token filtered."""
        import torch
        q = self._check_q(queries)
        B = int(q.shape[0])
        if not probes.is_cuda or probes.dtype != torch.int32 or probes.dim() != 2 or \
                probes.shape[0] != B:
            raise TypeError("probes must be an int32 GPU tensor [B, S]")
        pr = probes.contiguous()
        nt = self._next_tok(next_tok, B)
        idx, score, tok = _search_out(B, k, self.L, tokens, q.device, out)
        _lib.check(self._lib.dresd_ivf_search_probes(
            self._h, ctypes.c_void_p(q.data_ptr()), ctypes.c_void_p(pr.data_ptr()),
            int(pr.shape[1]), ctypes.c_void_p(nt.data_ptr()) if nt is not None else None, B,
            int(k), ctypes.c_void_p(idx.data_ptr()), ctypes.c_void_p(score.data_ptr()),
            ctypes.c_void_p(tok.data_ptr()) if tok is not None else None, _stream_handle(stream)))
        return idx, score, tok

    def info(self):
        N, d, L, dt, P, T = (ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32(),
                             ctypes.c_int32(), ctypes.c_int64())
        _lib.check(self._lib.dresd_ivf_info(self._h, ctypes.byref(N), ctypes.byref(d),
                                            ctypes.byref(L), ctypes.byref(dt), ctypes.byref(P),
                                            ctypes.byref(T)))
        return {"N": N.value, "d": d.value, "L": L.value, "dtype": dt.value, "P": P.value,
                "tiles": T.value}

    def profile(self, on: bool = True):
        _lib.check(self._lib.dresd_ivf_profile_enable(self._h, 1 if on else 0))

    def profile_read(self):
        a, b, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_int64()
        _lib.check(self._lib.dresd_ivf_profile_read(self._h, ctypes.byref(a), ctypes.byref(b),
                                                    ctypes.byref(n)))
        return {"scan_ms": a.value, "search_ms": b.value, "searches": n.value}

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self._lib.dresd_ivf_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def transform(x, mean, var, W, eps_z: float = 1e-5, eps_n: float = 1e-12, out=None, stream=None):
    """Query-side transform of Algorithm 1 steps 4-6 on the GPU: z-score
    normalisation (Eq. 1), projection onto the principal components W
    ([D, l], Section 3.3) and L2 normalisation (Eq. 2).  All tensors are
    float32 on the GPU; returns y [M, l]."""
    import torch
    for name, t in (("x", x), ("mean", mean), ("var", var), ("W", W)):
        if not t.is_cuda or t.dtype != torch.float32:
            raise TypeError("%s must be a float32 GPU tensor" % name)
    if x.dim() != 2 or W.dim() != 2 or W.shape[0] != x.shape[1]:
        raise ValueError("x must be [M, D] and W [D, l]")
    M, D = int(x.shape[0]), int(x.shape[1])
    l = int(W.shape[1])
    if mean.numel() != D or var.numel() != D:
        raise ValueError("mean and var must hold D values")
    x, mean, var, W = x.contiguous(), mean.contiguous(), var.contiguous(), W.contiguous()
    y = torch.empty((M, l), dtype=torch.float32, device=x.device) if out is None else out
    lib = _lib.load()
    _lib.check(lib.dresd_transform(ctypes.c_void_p(x.data_ptr()), M, D,
                                   ctypes.c_void_p(mean.data_ptr()),
                                   ctypes.c_void_p(var.data_ptr()), float(eps_z),
                                   ctypes.c_void_p(W.data_ptr()), l, float(eps_n),
                                   ctypes.c_void_p(y.data_ptr()), _stream_handle(stream)))
    return y


def pack_drafts(tokens, r: int, length: int, eos: int = 0, out=None, stream=None):
    """Draft assembly for batch verification (Section 3.6) on the GPU: tokens
    [B, k, L] int32 (from ``Index.search``) -> (drafts [B, r, length] int32,
    count [B] int32): EOS-padded rows, drafts starting with EOS and repeats
    dropped in rank order."""
    import torch
    if not tokens.is_cuda or tokens.dtype != torch.int32 or tokens.dim() != 3:
        raise TypeError("tokens must be an int32 GPU tensor [B, k, L]")
    B, k, L = (int(s) for s in tokens.shape)
    t = tokens.contiguous()
    if out is None:
        drafts = torch.empty((B, r, length), dtype=torch.int32, device=t.device)
        count = torch.empty((B,), dtype=torch.int32, device=t.device)
    else:
        drafts, count = out
    lib = _lib.load()
    _lib.check(lib.dresd_pack_drafts(ctypes.c_void_p(t.data_ptr()), B, k, L, int(r), int(length),
                                     int(eos), ctypes.c_void_p(drafts.data_ptr()),
                                     ctypes.c_void_p(count.data_ptr()), _stream_handle(stream)))
    return drafts, count


# ---- batch verification: the forward over the drafts, around the model's weights -----------


class _Here:
    """The context of a call whose device is current and whose stream is the current one."""

    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_HERE = _Here()


def _on(stream, *tensors):
    """Context in which a call on these GPU tensors allocates and launches: their device, and
    ``stream`` (outputs and workspaces then belong to it, and a later call on it may reuse
    them)."""
    import torch
    index = -1
    for t in tensors:
        if t is None:
            continue
        i = t.get_device()
        if i < 0:
            raise TypeError("all inputs must be GPU tensors")
        if index < 0:
            index = i
        elif i != index:
            raise ValueError("all tensors must be on one device")
    if stream is not None:
        if stream.device.index != index:
            raise ValueError("the stream must be on the tensors' device")
        return torch.cuda.stream(stream)
    if index != torch._C._cuda_getDevice():
        return torch.cuda.device(index)
    return _HERE


def _current(t):
    """Handle of the current stream of a tensor's device."""
    import torch
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _expect(name, t, dtype, *shape):
    """A contiguous tensor of this type and shape."""
    if t.dtype != dtype:
        raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, not %s" % (name, list(shape), list(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _expect_dim(name, t, dim):
    if t.dim() != dim:
        raise ValueError("%s must have %d dimensions" % (name, dim))
    return t.shape


def _ptr(t):
    return None if t is None else t.data_ptr()


def _too_far(what):
    """For sizes (all of them or-ed together) with a bit past the 31 that the C entry takes; ctypes
    would cut them."""
    raise ValueError("%s must fit 32 bits" % what)


def draft_tree(drafts, count, next_tok, nodes: int | None = None, eos: int = 0, out=None,
               stream=None):
    """Prefix tree of each query's drafts (Section 3.6), the tokens that one
    forward verifies: ``drafts`` [B, r, length] and ``count`` [B] int32 from
    ``pack_drafts``, ``next_tok`` [B] int32, the token they start with, which is
    node 0.  Draft by draft in rank order every new prefix is a node, up to
    ``nodes`` of them (default: as many as the shape can need, at most
    ``NODES_MAX``).  Returns (token [B, N], parent [B, N], depth [B, N] int32, mask
    [B, N, ceil(N / 64)] int64, nodes [B] int32): bit v of a node's mask row is
    set where v is the node or its ancestor (as ``paged_attention`` takes it),
    depth counts its tokens after node 0; past a query's last node the token is
    ``eos``, the parent -1, depth and mask 0."""
    import torch
    i32 = torch.int32
    B, r, length = _expect_dim("drafts", drafts, 3)
    _expect("drafts", drafts, i32, B, r, length)
    _expect("count", count, i32, B)
    _expect("next_tok", next_tok, i32, B)
    N = min(NODES_MAX, 1 + r * max(0, length - 1)) if nodes is None else int(nodes)
    if not 1 <= N <= NODES_MAX:
        raise ValueError("nodes must be in [1, %d]" % NODES_MAX)
    eos = int(eos)
    if (B | r | length) >> 31 or not -0x80000000 <= eos <= 0x7fffffff:
        _too_far("the shape of drafts and eos")
    W = (N + 63) // 64
    with _on(stream, drafts, count, next_tok, *(out or ())):
        if out is None:
            out = (*drafts.new_empty((3, B, N)).unbind(),
                   drafts.new_empty((B, N, W), dtype=torch.int64), torch.empty_like(count))
        else:
            for name, t in zip(("token", "parent", "depth"), out):
                _expect(name, t, i32, B, N)
            _expect("mask", out[3], torch.int64, B, N, W)
            _expect("nodes", out[4], i32, B)
        _lib.check(_lib.load().dresd_draft_tree(
            drafts.data_ptr(), count.data_ptr(), next_tok.data_ptr(), B, r, length, eos, N,
            *(t.data_ptr() for t in out), _current(drafts)))
    return tuple(out)


_CACHE_DTYPES = None


def _kv_cache(k_pages, v_pages, k_exp, v_exp):
    """The C description of a paged cache."""
    import torch
    global _CACHE_DTYPES
    if _CACHE_DTYPES is None:
        _CACHE_DTYPES = {torch.float16: _lib.F16, torch.bfloat16: _lib.BF16,
                         torch.float8_e4m3fn: _lib.F8}
    code = _CACHE_DTYPES.get(k_pages.dtype)
    if code is None:
        raise TypeError("a cache is float16, bfloat16 or float8_e4m3fn, not %s" % k_pages.dtype)
    P, H, page, D = shape = _expect_dim("k_pages", k_pages, 4)
    if (H | page | D) >> 31:
        _too_far("a cache's heads, page size and dim")
    # (one condition where all is well: a call of one token is bound by these checks)
    if not (v_pages.dtype == k_pages.dtype and v_pages.shape == shape and k_pages.is_contiguous()
            and v_pages.is_contiguous()):
        _expect("k_pages", k_pages, k_pages.dtype, P, H, page, D)
        _expect("v_pages", v_pages, k_pages.dtype, P, H, page, D)
    if code != _lib.F8:
        if k_exp is not None or v_exp is not None:
            raise ValueError("an 8-bit cache has k_exp and v_exp, a 16-bit one neither")
        return _lib.KvCache(k_pages.data_ptr(), v_pages.data_ptr(), None, None, P, page, H, D, code)
    if k_exp is None or v_exp is None:
        raise ValueError("an 8-bit cache has k_exp and v_exp, a 16-bit one neither")
    u8, exps = torch.uint8, (P, H, page)
    if not (k_exp.dtype == u8 == v_exp.dtype and k_exp.shape == exps == v_exp.shape
            and k_exp.is_contiguous() and v_exp.is_contiguous()):
        _expect("k_exp", k_exp, u8, P, H, page)
        _expect("v_exp", v_exp, u8, P, H, page)
    return _lib.KvCache(k_pages.data_ptr(), v_pages.data_ptr(), k_exp.data_ptr(),
                        v_exp.data_ptr(), P, page, H, D, code)


def kv_write(k, v, slots, k_pages, v_pages, k_exp=None, v_exp=None, stream=None) -> None:
    """Write tokens' keys and values ([n, heads, dim], float32, float16 or
    bfloat16; slices of a projection's output need no copy) into the slots
    (int64 [n]) of a paged cache: ``k_pages`` and ``v_pages`` [pages, heads,
    page_size, dim], slot s being row s % page_size of page s // page_size.  The
    cache is float16, bfloat16, or float8_e4m3fn with a power of two a row (one token
    of one head) in ``k_exp`` and ``v_exp`` (uint8 [pages, heads, page_size]): the
    row's values are the stored ones times 2 ** (exp - 127).  Tokens whose slot
    is outside the cache (-1, say) are skipped; two tokens must not share a slot."""
    import torch
    shape = k.shape
    if len(shape) != 3 or shape != v.shape or k.dtype != v.dtype:
        raise ValueError("k and v must be [n, heads, dim] of one type")
    n, heads, dim = shape
    cache = _kv_cache(k_pages, v_pages, k_exp, v_exp)
    if heads != cache.heads or dim != cache.dim:
        raise ValueError("k and v must be [n, %d, %d]" % (cache.heads, cache.dim))
    kr, kh, kd = k.stride()
    vr, vh, vd = v.stride()
    if kd != 1 or vd != 1:
        raise ValueError("the last dimension of k and v must be contiguous")
    if n < 2:                  # (strides that are never taken)
        kr = vr = 0
    if heads < 2:
        kh = vh = 0
    _expect("slots", slots, torch.int64, n)
    with _on(stream, k, v, slots, k_pages, v_pages, k_exp, v_exp):
        _lib.check(_lib.load().dresd_kv_write(
            cache, k.data_ptr(), kr, kh, v.data_ptr(), vr, vh, _dtype_code(k), slots.data_ptr(), n,
            _current(k)))


def kv_read(slots, k_pages, v_pages, k_exp=None, v_exp=None, dtype=None, out=None, stream=None):
    """Keys and values of cache slots (int64 [n], any order, repeats allowed;
    zeros for a slot outside the cache) as (k, v) [n, heads, dim] in ``dtype``
    (float32, float16 or bfloat16; default: the cache's, bfloat16 for 8-bit caches,
    which holds the values of their rows past 2 ** -116 exactly)."""
    import torch
    cache = _kv_cache(k_pages, v_pages, k_exp, v_exp)
    n, = _expect_dim("slots", slots, 1)
    _expect("slots", slots, torch.int64, n)
    if dtype is None:
        dtype = torch.bfloat16 if cache.dtype == _lib.F8 else k_pages.dtype
    with _on(stream, slots, k_pages, v_pages, k_exp, v_exp, *(out or ())):
        if out is None:
            k = slots.new_empty((n, cache.heads, cache.dim), dtype=dtype)
            out = (k, torch.empty_like(k))
        else:
            _expect("k", out[0], dtype, n, cache.heads, cache.dim)
            _expect("v", out[1], dtype, n, cache.heads, cache.dim)
        _lib.check(_lib.load().dresd_kv_read(
            cache, slots.data_ptr(), n, _dtype_code(out[0]), out[0].data_ptr(),
            out[1].data_ptr(), _current(slots)))
    return tuple(out)


@functools.lru_cache(maxsize=1024)
def _attention_workspace(device, pages, page, heads, dim, dtype, q_heads, ragged, n, B, T, width):
    """Bytes of workspace of a call of this shape (the device is current)."""
    need = ctypes.c_int64()
    _lib.check(_lib.load().dresd_paged_attention_workspace(
        _lib.KvCache(None, None, None, None, pages, page, heads, dim, dtype), q_heads, ragged, n,
        B, T, width, ctypes.byref(need)))
    return need.value


def paged_attention(q, k_pages, v_pages, table, lengths, starts=None, mask=None, k_exp=None,
                    v_exp=None, scale: float | None = None, with_lse: bool = False, out=None,
                    stream=None):
    """Attention of each sequence's newest tokens, its chunk (one decoded token, a
    draft tree, a piece of a prompt), over a paged cache that holds them already
    (``kv_write``).  Sequence b has ``lengths[b]`` (int32 [B]) tokens in the cache,
    the last of them its chunk, and its position p in page ``table[b, p // page_size]``
    (int32 [B, width]).  ``q`` (float16 or bfloat16, that of a 16-bit cache) is
    [B, n, q_heads, dim], or [T, q_heads, dim] with sequence b's chunk in rows
    ``starts[b]`` to ``starts[b + 1] - 1`` (int32 [B + 1]); query head h reads
    cache head h // (q_heads // heads).  A row sees the positions up to its own;
    with ``mask`` (int64 [B, n, words] or [T, words]; ``draft_tree``) all before the
    chunk and the chunk tokens whose bit is set.  ``scale`` defaults to dim ** -0.5.
    Returns the output, shaped as q and in its type (zeros for a row that sees
    nothing; rows outside every chunk are left as they were; no gradient), and with ``with_lse``
    also the fp32 logarithms of the rows' sums ([..., q_heads]; -inf for a row
    that sees nothing).  ``out``: the output tensor, or the pair."""
    import torch
    cache = _kv_cache(k_pages, v_pages, k_exp, v_exp)
    B, = _expect_dim("lengths", lengths, 1)
    width = _expect_dim("table", table, 2)[1]
    _expect("lengths", lengths, torch.int32, B)
    _expect("table", table, torch.int32, B, width)
    if q.dtype not in (torch.float16, torch.bfloat16):
        raise TypeError("q must be float16 or bfloat16, not %s" % q.dtype)
    shape, strides = q.shape, q.stride()
    if starts is None:
        if len(shape) != 4 or shape[0] != B:
            raise ValueError("without starts q must be [%d, n, q_heads, dim]" % B)
        n = shape[1]
        T, row = B * n, strides[1 if n > 1 else 0]
        if n > 1 and B > 1 and strides[0] != n * strides[1]:
            raise ValueError("q's tokens must be evenly spaced")
    else:
        _expect("starts", starts, torch.int32, B + 1)
        if len(shape) != 3:
            raise ValueError("with starts q must be [T, q_heads, dim]")
        n, T, row = 0, shape[0], strides[0]
    H = shape[-2]
    if shape[-1] != cache.dim or strides[-1] != 1:
        raise ValueError("q's last dimension must be %d contiguous elements" % cache.dim)
    head = strides[-2] if H > 1 else 0           # (0: a stride that is never taken)
    if T < 2:
        row = 0
    words = 0
    if mask is not None:
        words = _expect_dim("mask", mask, q.dim() - 1)[-1]
        if words < 1:          # (an empty tensor has no address, which is no mask)
            raise ValueError("mask must have a word a row at least")
        _expect("mask", mask, torch.int64, *q.shape[:-2], words)
    if (n | B | H | width | words) >> 31:
        _too_far("the shapes of q, table and mask")
    if scale is None:
        scale = cache.dim ** -0.5
    given = out if isinstance(out, (tuple, list)) else () if out is None else (out,)
    lib = _lib.load()
    with _on(stream, q, k_pages, v_pages, k_exp, v_exp, table, lengths, starts, mask, *given):
        if not given:
            o = q.new_empty(q.shape)
            lse = q.new_empty(q.shape[:-1], dtype=torch.float32) if with_lse else None
        else:
            o, lse = given[0], given[1] if len(given) > 1 else None
            if (lse is not None) != with_lse:
                raise ValueError("out must be the pair exactly with with_lse")
            _expect("out", o, q.dtype, *q.shape)
            if lse is not None:
                _expect("lse", lse, torch.float32, *q.shape[:-1])
        need = _attention_workspace(q.get_device(), cache.pages, cache.page_size, cache.heads,
                                    cache.dim, cache.dtype, H, starts is not None, n, B, T, width)
        work = q.new_empty((need,), dtype=torch.uint8) if need else None
        _lib.check(lib.dresd_paged_attention(
            cache, q.data_ptr(), row, head, _dtype_code(q), H, _ptr(starts), n, B, T,
            table.data_ptr(), width, lengths.data_ptr(), _ptr(mask), words, float(scale),
            o.data_ptr(), _ptr(lse), _ptr(work), need, _current(q)))
    return (o, lse) if with_lse else o


def accept_drafts(logits, token, parent, nodes, most: int | None = None, out=None, stream=None):
    """Acceptance of a draft tree (``draft_tree``'s token, parent [B, N] and nodes
    [B]) by the model's own greedy tokens: from node 0, on to the child that holds
    the token of the node's largest logit (ties to the lower token), while there
    is one and fewer than ``most`` (default N) nodes are accepted.  ``logits``
    [B, N, V] float32, float16 or bfloat16, rows evenly spaced and apart (slices of
    padded rows need no copy, expanded ones do).  Returns (path [B, most] int32:
    the accepted nodes, then -1; accepted [B] int32: their number; next_tok [B]
    int32: the model's token after the last of them)."""
    import torch
    i32 = torch.int32
    if logits.dim() != 3:
        raise ValueError("logits must be [B, N, V]")
    B, N, V = logits.shape
    sb, sn, sv = logits.stride()
    row = V if B * N < 2 else sn if N > 1 else sb    # (one row: its stride is never taken)
    if sv != 1 and V > 1 or row < V or (N > 1 and B > 1 and sb != N * row):
        raise ValueError("the rows of logits must be contiguous, evenly spaced and apart")
    _expect("token", token, i32, B, N)
    _expect("parent", parent, i32, B, N)
    _expect("nodes", nodes, i32, B)
    most = N if most is None else int(most)
    if (B | N | V | most) >> 31:
        _too_far("the shape of logits and most")
    with _on(stream, logits, token, parent, nodes, *(out or ())):
        if out is None:
            out = (token.new_empty((B, most)), *token.new_empty((2, B)).unbind())
        else:
            _expect("path", out[0], i32, B, most)
            _expect("accepted", out[1], i32, B)
            _expect("next_tok", out[2], i32, B)
        _lib.check(_lib.load().dresd_accept_drafts(
            logits.data_ptr(), _dtype_code(logits), row, V, token.data_ptr(),
            parent.data_ptr(), nodes.data_ptr(), B, N, most, *(t.data_ptr() for t in out),
            _current(logits)))
    return tuple(out)


def _rows(x):
    if not x.is_cuda or x.dim() != 2:
        raise TypeError("rows must be a GPU tensor [n, d]")
    return x.contiguous()


def kmeans_assign(x, centroids, with_score: bool = False, stream=None):
    """Nearest centroid by inner product for every row of ``x`` ([n, d],
    float32/float16/bfloat16 on the GPU; ``centroids`` float32 [P, d]), ties
    to the lower id.  Returns assign int32 [n] (and the fp32 scores)."""
    import torch
    x = _rows(x)
    c = centroids.contiguous()
    if c.dtype != torch.float32 or c.dim() != 2 or c.shape[1] != x.shape[1]:
        raise TypeError("centroids must be float32 [P, d]")
    n, d = int(x.shape[0]), int(x.shape[1])
    a = torch.empty((n,), dtype=torch.int32, device=x.device)
    sc = torch.empty((n,), dtype=torch.float32, device=x.device) if with_score else None
    _lib.check(_lib.load().dresd_kmeans_assign(
        ctypes.c_void_p(x.data_ptr()), n, d, _dtype_code(x), ctypes.c_void_p(c.data_ptr()),
        int(c.shape[0]), ctypes.c_void_p(a.data_ptr()),
        ctypes.c_void_p(sc.data_ptr()) if sc is not None else None, _stream_handle(stream)))
    return (a, sc) if with_score else a


def kmeans_update(x, assign, centroids, stream=None):
    """Spherical k-means update in place: each centroid (float32 [P, d],
    contiguous) becomes the unit vector along the sum of its rows (unchanged
    without rows).  Returns the rows per centroid (int32 [P])."""
    import torch
    x = _rows(x)
    if not centroids.is_contiguous() or centroids.dtype != torch.float32:
        raise TypeError("centroids must be a contiguous float32 tensor [P, d]")
    if assign.dtype != torch.int32 or assign.numel() != x.shape[0]:
        raise TypeError("assign must be int32 with one entry per row")
    a = assign.contiguous()
    P = int(centroids.shape[0])
    counts = torch.empty((P,), dtype=torch.int32, device=x.device)
    _lib.check(_lib.load().dresd_kmeans_update(
        ctypes.c_void_p(x.data_ptr()), int(x.shape[0]), int(x.shape[1]), _dtype_code(x),
        ctypes.c_void_p(a.data_ptr()), P, ctypes.c_void_p(centroids.data_ptr()),
        ctypes.c_void_p(counts.data_ptr()), _stream_handle(stream)))
    return counts


def kmeans_init(x, P: int, seed: int = 0, stream=None):
    """Starting centroids of spherical k-means (float32 [P, d]): P distinct
    rows of ``x`` at even spacing through the row order from an offset drawn
    from ``seed`` (SplitMix64), each scaled to unit length."""
    import torch
    x = _rows(x)
    n, d = int(x.shape[0]), int(x.shape[1])
    if not (1 <= P <= n):
        raise ValueError("need 1 <= P <= n")
    if not (0 <= seed < 1 << 64):
        raise ValueError("seed must be in [0, 2^64)")
    centroids = torch.empty((P, d), dtype=torch.float32, device=x.device)
    _lib.check(_lib.load().dresd_kmeans_init(
        ctypes.c_void_p(x.data_ptr()), n, d, _dtype_code(x), P, seed,
        ctypes.c_void_p(centroids.data_ptr()), _stream_handle(stream)))
    return centroids


def train_partitions(x, P: int, iters: int = 10, seed: int = 0, stream=None):
    """Spherical k-means on the GPU: P centroids started by kmeans_init, then
    ``iters`` assign + update steps.  Returns (centroids float32 [P, d],
    assign int32 [n])."""
    x = _rows(x)
    centroids = kmeans_init(x, P, seed, stream)
    for _ in range(iters):
        assign = kmeans_assign(x, centroids, stream=stream)
        kmeans_update(x, assign, centroids, stream)
    return centroids, kmeans_assign(x, centroids, stream=stream)


def release_cached() -> None:
    """Give back the device memory that the library holds for later calls
    (large blocks of closed indexes, operand and sorting buffers), for a program
    whose other allocators need it.  Not while a stream is being captured."""
    _lib.check(_lib.load().dresd_release_cached())


def bw_probe(buf, reps: int = 10, workgroups: int = 0, stream=None) -> float:
    """Achievable HBM read bandwidth with the scans' access pattern: reads
    every byte of the GPU tensor ``buf`` (contents irrelevant; whole 1 KiB
    blocks, at least 1 MiB) ``reps`` times after one untimed pass with
    ``workgroups`` workgroups (0: four per compute unit).  Returns GB/s."""
    if not buf.is_cuda:
        raise ValueError("buf must be a GPU tensor")
    nbytes = buf.numel() * buf.element_size() // 1024 * 1024
    lib = _lib.load()
    ms = ctypes.c_double()
    _lib.check(lib.dresd_bw_probe(ctypes.c_void_p(buf.data_ptr()), nbytes, int(reps),
                                  int(workgroups), ctypes.byref(ms), _stream_handle(stream)))
    return nbytes / (ms.value * 1e-3) / 1e9
