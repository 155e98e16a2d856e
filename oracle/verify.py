"""Plain oracle of batch verification's operators (numpy, 64 bits): prefix trees
of drafts, cache rows in 8 bits, attention of chunks over a cache, acceptance.
Written from the definitions, one token at a time."""
from __future__ import annotations

import numpy as np


def draft_tree(drafts, count, next_tok, N, eos=0):
    """(token [B, N], parent, depth, ancestors: list of sets per node, nodes [B])."""
    B, r, _ = drafts.shape
    token = np.full((B, N), eos, np.int32)
    parent = np.full((B, N), -1, np.int32)
    depth = np.zeros((B, N), np.int32)
    nodes = np.zeros(B, np.int32)
    anc = []
    for b in range(B):
        known = {(): 0}          # prefix after node 0 -> node
        token[b, 0] = next_tok[b]
        sets = [{0}]
        for i in range(min(max(int(count[b]), 0), r)):
            d = drafts[b, i].tolist()
            if eos in d:
                d = d[:d.index(eos)]
            if not d or d[0] != next_tok[b]:
                continue
            for p in range(1, len(d)):
                prefix = tuple(d[1:p + 1])
                if prefix in known:
                    continue
                u = len(sets)
                if u >= N:
                    break
                known[prefix] = u
                up = known[prefix[:-1]]
                token[b, u], parent[b, u], depth[b, u] = d[p], up, p
                sets.append(sets[up] | {u})
        nodes[b] = len(sets)
        anc.append(sets)
    return token, parent, depth, anc, nodes


def mask_words(anc, N):
    """Ancestor sets as [B, N, W] uint64 bits."""
    W = (N + 63) // 64
    out = np.zeros((len(anc), N, W), np.uint64)
    for b, sets in enumerate(anc):
        for u, s in enumerate(sets):
            for v in s:
                out[b, u, v // 64] |= np.uint64(1) << np.uint64(v % 64)
    return out


# every non-negative finite e4m3 value, by code
E4M3 = np.array([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
                 for e in range(16) for m in range(8)][:127])


def e4m3(x):
    """Codes of values of at most 448, nearest, ties to the even code; NaN is 0x7f."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isnan(x), 0.0, np.abs(x))
    hi = np.clip(np.searchsorted(E4M3, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dh, dl = E4M3[hi] - a, a - E4M3[lo]
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(a == E4M3[hi], hi, c)
    return np.where(np.isnan(x), 0x7f, c | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def e4m3_value(code):
    code = np.asarray(code, np.uint8)
    c = code & 127
    v = np.where(c == 127, np.nan, E4M3[np.minimum(c, 126)])
    return np.where(code >> 7, -v, v)


def quantise(x):
    """Rows x [..., dim] -> (codes uint8, exponent bytes uint8)."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isfinite(x), x, np.nan)
    top = np.nanmax(np.where(np.isnan(x), 0.0, np.abs(x)), axis=-1)
    e = np.empty(top.shape, np.int64)
    for i in np.ndindex(top.shape):
        e[i] = -9
        if top[i] > 0:
            e[i] = -126
            while top[i] > 448.0 * 2.0 ** float(e[i]):
                e[i] += 1
    # at the top of fp32 a value rounded up to 2^128 could not be read back: the code below it
    most = np.where(e == 120, 240.0, 448.0)[..., None]
    y = np.clip(x * 2.0 ** -e[..., None].astype(np.float64), -most, most)
    return e4m3(y), (e + 127).astype(np.uint8)


def dequantise(codes, exp):
    return e4m3_value(codes) * 2.0 ** (np.asarray(exp, np.float64) - 127.0)[..., None]


def attend(q, k, v, see, scale):
    """q [n, H, D], k, v [L, hk, D] float64, see [n, L] -> (out [n, H, D], lse [n, H], the sum of
    the weighted magnitudes [n, H, D], and the sum of |q||k| of the row's largest score [n, H]).
    Positions that a row does not see take no part, whatever they hold."""
    n, H, D = q.shape
    G = H // k.shape[1] if k.shape[1] else 1
    out, mag = np.zeros((n, H, D)), np.zeros((n, H, D))
    lse, size = np.full((n, H), -np.inf), np.zeros((n, H))
    for t in range(n):
        w = np.nonzero(see[t])[0]
        if not w.size:
            continue
        for h in range(H):
            kk, vv = k[w, h // G], v[w, h // G]
            s = scale * (kk @ q[t, h])
            m = s.max()
            p = np.exp(s - m)
            lse[t, h] = m + np.log(p.sum())
            p = p / p.sum()
            out[t, h] = p @ vv
            mag[t, h] = p @ np.abs(vv)
            size[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out, lse, mag, size


def accept(logits, token, parent, nodes, most):
    """(path [B, most], accepted [B], next_tok [B])."""
    B, N, V = logits.shape
    path = np.full((B, most), -1, np.int32)
    accepted, nxt = np.zeros(B, np.int32), np.full(B, -1, np.int32)
    for b in range(B):
        n = min(max(int(nodes[b]), 0), N)
        u = 0 if n > 0 else -1
        while u >= 0:
            path[b, accepted[b]] = u
            accepted[b] += 1
            row = logits[b, u]
            g = 0 if np.isnan(row).all() else int(np.nanargmax(row))
            nxt[b] = g
            u = next((c for c in range(u + 1, n)
                      if accepted[b] < most and parent[b, c] == u and token[b, c] == g), -1)
    return path, accepted, nxt
