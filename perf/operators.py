"""The operators of the verifying forward, one case per use of them.

A program that decodes with retrieved drafts runs, at every step, one forward of
its language model over the drafts.  The drafts become a prefix tree; in each
layer the keys and values of the tree's tokens are written into a paged cache and
its queries attend over the cached context and their own ancestors; the logits of
the tree's nodes decide which path is accepted; the accepted tokens' entries are
read and written to their final slots.  The same cache serves prompts, written and
attended chunk by chunk, and single tokens where no draft was found.

listed() are the cases, draw() makes more of the same ranges.  prepare() makes
what a program holds before the call, run() is one call, exact() the same result
in 64 bits from plain torch.
"""
import math

import torch

own = False

DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16,
      "f8": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "f8": 1}
VOCAB = 32000        # tokens of the models whose hidden states the datastores hold
EOS = 0


def listed():
    return [
        # One sequence, one step's ten drafts: all latency.
        {"name": "tree_b1", "kind": "tree", "B": 1, "r": 10, "length": 10, "N": 91},
        # A serving batch with every retrieved continuation kept, cut at a budget of nodes.
        {"name": "tree_b128", "kind": "tree", "B": 128, "r": 100, "length": 20, "N": 1000},
        # One decoded token of each sequence enters an 8-bit cache: all latency.
        {"name": "write_step_f8", "kind": "write", "dtype": "bf16", "cache": "f8", "n": 48,
         "heads": 8, "dim": 128, "page": 16, "pages": 2048},
        # A chunk of prompt tokens enters an 8-bit cache, every head with its own keys.
        {"name": "write_prompt_f8", "kind": "write", "dtype": "bf16", "cache": "f8", "n": 16384,
         "heads": 32, "dim": 128, "page": 64, "pages": 512},
        # The accepted paths of a batch are moved within an 8-bit cache.
        {"name": "read_path_f8", "kind": "read", "dtype": "bf16", "cache": "f8", "n": 77,
         "heads": 8, "dim": 128, "page": 16, "pages": 2048},
        # A long sequence is taken out of the cache, ragged width and page.
        {"name": "read_sequence_f16", "kind": "read", "dtype": "f32", "cache": "f16", "n": 50001,
         "heads": 12, "dim": 80, "page": 32, "pages": 2000},
        # One sequence without a draft: one token over a long context, grouped heads.
        {"name": "attend_step_b1", "kind": "attend", "dtype": "bf16", "cache": "bf16", "B": 1,
         "n": 1, "ctx": 32001, "heads": 8, "group": 4, "dim": 128, "page": 16, "tree": False,
         "ragged": False, "lse": False},
        # A serving batch's single tokens over ragged contexts in an 8-bit cache.
        {"name": "attend_step_f8_b64", "kind": "attend", "dtype": "bf16", "cache": "f8", "B": 64,
         "n": 1, "ctx": 8000, "heads": 8, "group": 8, "dim": 128, "page": 64, "tree": False,
         "ragged": False, "lse": False},
        # Verification: the draft trees of a batch, every head with its own keys.
        {"name": "attend_tree_f16_b8", "kind": "attend", "dtype": "f16", "cache": "f16", "B": 8,
         "n": 91, "ctx": 4000, "heads": 32, "group": 1, "dim": 128, "page": 16, "tree": True,
         "ragged": False, "lse": True},
        # Chunks of three prompts over what is cached of them.
        {"name": "attend_prompt_bf16", "kind": "attend", "dtype": "bf16", "cache": "bf16", "B": 3,
         "n": 2048, "ctx": 16000, "heads": 8, "group": 4, "dim": 128, "page": 64, "tree": False,
         "ragged": True, "lse": False},
        # One sequence's ten drafts are judged.
        {"name": "accept_b1", "kind": "accept", "dtype": "f32", "B": 1, "r": 10, "length": 10,
         "N": 91, "V": VOCAB},
        # A batch's trees over a large vocabulary.
        {"name": "accept_b64", "kind": "accept", "dtype": "bf16", "B": 64, "r": 10, "length": 8,
         "N": 64, "V": 128000},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "write", "read", "attend", "attend", "attend", "attend", "accept"])
    if kind == "tree":
        r, length = _log(rng, 1, 100), _log(rng, 2, 20)
        full = 1 + r * (length - 1)
        return {"kind": kind, "B": _log(rng, 1, 128), "r": r, "length": length,
                "N": rng.choice([min(full, 1000), max(1, min(full, _log(rng, 8, 1000)))])}
    dtype = rng.choice(["f16", "bf16"])
    if kind == "accept":
        B = _log(rng, 1, 64)
        r, length = _log(rng, 1, 20), _log(rng, 2, 12)
        return {"kind": kind, "dtype": rng.choice([dtype, "f32"]), "B": B, "r": r,
                "length": length, "N": min(1 + r * (length - 1), 64 if B > 8 else 256),
                "V": rng.choice([VOCAB, _log(rng, 1000, 64000)])}
    heads, dim = rng.choice([1, 2, 4, 8, 8, 12, 32]), rng.choice([64, 80, 96, 128, 128, 256])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    cache = rng.choice([dtype, "f8"])
    if kind in ("write", "read"):
        n = _log(rng, 1, min(50001, (1 << 26) // (heads * dim)))
        return {"kind": kind, "dtype": rng.choice([dtype, "f32"]), "cache": cache, "n": n,
                "heads": heads, "dim": dim, "page": page,
                "pages": max(8, int(n * rng.uniform(1.1, 1.5)) // page + 1)}
    use = rng.choice(["step", "step", "tree", "prompt"])
    heads = min(heads, 16)
    group = rng.choice([1, 2, 4, 4, 7, 8])
    if use == "step":
        B, n, ctx = _log(rng, 1, 64), 1, _log(rng, 1, 32000)
    elif use == "tree":
        B, n, ctx = _log(rng, 1, 16), _log(rng, 2, 128), _log(rng, 16, 8000)
    else:
        B, n, ctx = _log(rng, 1, 4), _log(rng, 16, 2048), _log(rng, 1, 16000)
    # no more cached values and no more scores than the largest listed cases have
    ctx = max(1, min(ctx, (1 << 28) // (B * heads * dim)))
    group = max(1, min(group, (3 << 29) // (B * heads * n * (ctx + n))))
    return {"kind": kind, "dtype": dtype, "cache": cache, "B": B, "n": n, "ctx": ctx,
            "heads": heads, "group": group, "dim": dim, "page": page, "tree": use == "tree",
            "ragged": use == "prompt", "lse": rng.random() < 0.3}


# ---- inputs ---------------------------------------------------------------------------------


def _gen(seed, part):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 64 + part)
    return g


def _randint(lo, hi, shape, g):
    return torch.randint(lo, hi, shape, device=DEV, generator=g)


def _drafts(case, seed):
    """Drafts that start with the next token, most of them leaving an earlier draft somewhere;
    every seventh ends early; the first one is whole.  Repeats of a draft are possible."""
    B, r, length = case["B"], case["r"], case["length"]
    g = _gen(seed, 0)
    d = _randint(1, VOCAB, (B, r, length), g)
    of = (torch.rand(B, r, device=DEV, generator=g) * torch.arange(r, device=DEV).clamp(min=1))
    of = of.to(torch.int64).clamp(max=max(0, r - 1))
    keep = _randint(1, length + 1, (B, r), g)
    at = torch.arange(length, device=DEV)
    # of the first draft, then of a draft that left it
    for _ in range(2):
        d = torch.where(at < keep[:, :, None], d.gather(1, of[:, :, None].expand(-1, -1, length)),
                        d)
    d[:, :, 0] = d[:, :1, 0]
    end = torch.where(_randint(0, 7, (B, r), g) == 0, _randint(1, length + 1, (B, r), g), length)
    end[:, 0] = length
    d = torch.where(at < end[:, :, None], d, EOS).to(torch.int32)
    count = _randint(max(1, r // 2), r + 1, (B,), g).to(torch.int32)
    d = torch.where(torch.arange(r, device=DEV)[None, :, None] < count[:, None, None], d, EOS)
    return d.to(torch.int32).contiguous(), count, d[:, 0, 0].to(torch.int32).contiguous()


def _rows(n, heads, dim, g):
    """Keys or values as a model makes them: every channel with its own scale, a few of them
    large, and every row with its own norm."""
    scale = torch.exp(0.7 * torch.randn(heads, dim, device=DEV, generator=g))
    size = torch.exp(0.3 * torch.randn(n, heads, 1, device=DEV, generator=g))
    x = torch.randn(n, heads, dim, device=DEV, generator=g)
    return x.mul_(scale).mul_(size)


def _exponents(x):
    """Each row's power of two: the smallest at which its largest value is at most 448."""
    f, e = torch.frexp(x.abs().amax(-1))
    return (e - 9 + (f > 0.875).to(e.dtype)).clamp(min=-126)


def _power(e):
    """2 ** e as float32, for exponents of -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _cache(case, pages, seed, part):
    """A filled cache: pages [pages, heads, page, dim] and, in 8 bits, the rows' exponents."""
    g = _gen(seed, part)
    heads, dim, page = case["heads"], case["dim"], case["page"]
    x = torch.empty(pages, heads, page, dim, dtype=DT[case["cache"]], device=DEV)
    f8 = case["cache"] == "f8"
    exp = torch.zeros(pages, heads, page, dtype=torch.uint8, device=DEV) if f8 else None
    step = max(1, (1 << 27) // (heads * page * dim))
    for a in range(0, pages, step):
        n = min(step, pages - a)
        y = _rows(n * page, heads, dim, g).view(n, page, heads, dim).transpose(1, 2).contiguous()
        if f8:
            e = _exponents(y)
            exp[a:a + n] = (e + 127).to(torch.uint8)
            y.mul_(_power(-e)[..., None])
        x[a:a + n] = y.to(x.dtype)
    return x, exp


def _lengths(case, seed):
    """Tokens of each sequence, the chunk's included, and the first rows of their chunks."""
    B, n, ctx = case["B"], case["n"], case["ctx"]
    at = torch.arange(B, dtype=torch.float64)
    # contexts between a quarter and the whole of ctx, chunks of ragged batches down to a half
    ctxs = (ctx * (1.0 - 0.75 * ((at * 0.618) % 1.0))).to(torch.int64).clamp(min=1)
    ns = (n * (1.0 - 0.5 * ((at * 0.381) % 1.0))).to(torch.int64).clamp(min=1) if case["ragged"] \
        else torch.full((B,), n, dtype=torch.int64)
    return (ctxs + ns).tolist(), ns.tolist()


def _visible_bits(case, seed):
    """Every node sees its ancestors and itself: [B, N, words] int64."""
    tree = {"B": case["B"], "r": max(1, -(-(case["n"] - 1) // 9)), "length": 10, "N": case["n"]}
    return _plain_tree(*_drafts(tree, seed), tree["N"])[3]


def _inputs(case, seed):
    kind = case["kind"]
    s = {"case": case}
    if kind == "tree":
        s["drafts"], s["count"], s["first"] = _drafts(case, seed)
    elif kind == "accept":
        B, N, V, length = case["B"], case["N"], case["V"], case["length"]
        d, count, first = _drafts(case, seed)
        d = torch.where(d == EOS, d, d % (V - 1) + 1)
        first = d[:, 0, 0].contiguous()
        s["token"], s["parent"], _, s["mask"], s["nodes"] = _plain_tree(d, count, first, N)
        g = _gen(seed, 1)
        logits = torch.empty(B, N, V, dtype=DT[case["dtype"]], device=DEV)
        for b in range(B):
            logits[b] = torch.randn(N, V, device=DEV, generator=g)
        # the model goes along the first draft, for a number of tokens that differs by sequence
        go = torch.tensor(_accepted(case), device=DEV)
        u = torch.arange(length - 1, device=DEV)
        nxt = d[:, 0, 1:].to(torch.int64)
        b, j = torch.nonzero(u < (go - 1)[:, None], as_tuple=True)
        logits[b, j, nxt[b, j]] = 20.0
        s["logits"] = logits
    elif kind in ("write", "read"):
        heads, dim, n = case["heads"], case["dim"], case["n"]
        s["k_pages"], s["k_exp"] = _cache(case, case["pages"], seed, 2)
        s["v_pages"], s["v_exp"] = _cache(case, case["pages"], seed, 3)
        s["slots"] = torch.randperm(case["pages"] * case["page"], device=DEV,
                                    generator=_gen(seed, 4))[:n]
        if n > 64:      # long runs of tokens lie in whole pages
            p = torch.randperm(case["pages"], device=DEV, generator=_gen(seed, 4))
            i = torch.arange(n, device=DEV)
            s["slots"] = p[i // case["page"]] * case["page"] + i % case["page"]
        if kind == "write":
            # the projection's output: queries, keys and values of a token side by side
            g = _gen(seed, 5)
            kv = torch.cat([_rows(n, heads, dim, g) for _ in range(2)], 1).to(DT[case["dtype"]])
            s["k"], s["v"] = kv[:, :heads], kv[:, heads:]
    else:
        B, heads, dim, page = case["B"], case["heads"], case["dim"], case["page"]
        H = heads * case["group"]
        lengths, ns = _lengths(case, seed)
        width = -(-max(lengths) // page)
        used = [-(-x // page) for x in lengths]
        pages = sum(used) + 3
        s["k_pages"], s["k_exp"] = _cache(case, pages, seed, 2)
        s["v_pages"], s["v_exp"] = _cache(case, pages, seed, 3)
        # pages in the order in which an allocator that has run for a while gives them out
        free = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))
        table = torch.zeros(B, width, dtype=torch.int32)
        for b in range(B):
            table[b, :used[b]] = free[sum(used[:b]):sum(used[:b + 1])]
        s["table"] = table.to(DEV)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        s["longest"], s["most"] = max(lengths), max(ns)
        T = sum(ns)
        starts = torch.tensor([0] + ns, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)
        # scores of a few units, as trained heads give
        qkv = _rows(T, H + 2, dim, _gen(seed, 6)).mul_(0.6).to(DT[case["dtype"]])
        q = qkv[:, :H]
        s["q"], s["starts"] = (q, starts) if case["ragged"] else (
            qkv.view(B, case["n"], H + 2, dim)[:, :, :H], None)
        s["rows"] = starts
        s["mask"] = _visible_bits(case, seed) if case["tree"] else None
    return s


def _accepted(case):
    """Nodes of the accepted path, by sequence."""
    most = min(case["length"], case["N"])
    return [1 + (3 * b + 2) % most for b in range(case["B"])]


def prepare(case, seed):
    return _inputs(case, seed)


# ---- the call -------------------------------------------------------------------------------


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _RUN[kind](s)
    return _PLAIN[kind](s)


def _run_tree(s):
    import paper_2502_15572_amd as dresd
    return dresd.draft_tree(s["drafts"], s["count"], s["first"], s["case"]["N"], EOS)


def _run_write(s):
    import paper_2502_15572_amd as dresd
    dresd.kv_write(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"])
    return s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"]


def _run_read(s):
    import paper_2502_15572_amd as dresd
    return dresd.kv_read(s["slots"], s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"],
                         dtype=DT[s["case"]["dtype"]])


def _run_attend(s):
    import paper_2502_15572_amd as dresd
    return dresd.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"],
                                 starts=s["starts"], mask=s["mask"], k_exp=s["k_exp"],
                                 v_exp=s["v_exp"], with_lse=s["case"]["lse"])


def _run_accept(s):
    import paper_2502_15572_amd as dresd
    return dresd.accept_drafts(s["logits"], s["token"], s["parent"], s["nodes"],
                               s["case"]["length"])


_RUN = {"tree": _run_tree, "write": _run_write, "read": _run_read, "attend": _run_attend,
        "accept": _run_accept}


# ---- plain forms ----------------------------------------------------------------------------


def _plain_tree(drafts, count, first, N):
    B, r, length = drafts.shape
    i, p = torch.arange(r, device=DEV), torch.arange(length, device=DEV)
    lens = (drafts != EOS).to(torch.int32).cumprod(2).sum(2)
    lens = torch.where((i < count[:, None]) & (drafts[:, :, 0] == first[:, None]), lens, 0)
    real = p < lens[:, :, None]
    same = (drafts[:, :, None] == drafts[:, None]) & real[:, :, None] & real[:, None]
    lcp = same.to(torch.int32).cumprod(3).sum(3)                         # [B, r, r]
    seen = torch.where(i[None, :] < i[:, None], lcp, 0).amax(2).clamp(min=1)
    new = (lens - seen).clamp(min=0)
    base = 1 + new.cumsum(1) - new
    # the first draft that holds the prefix of draft i up to p, and the prefix's node
    holds = (lcp[:, :, :, None] > p) & (i[None, :] <= i[:, None])[None, :, :, None]
    j = torch.where(holds, i[None, None, :, None], r - 1).amin(2)        # [B, r, length]
    node = base.gather(1, j.view(B, -1)).view(j.shape) + p - seen.gather(
        1, j.view(B, -1)).view(j.shape)
    node = torch.where(p == 0, 0, node)
    fresh = real & (p >= seen[:, :, None]) & (node < N)
    at = torch.where(fresh, node, N).view(B, -1)                         # past the budget: dropped
    up = torch.cat([node[:, :, :1], node[:, :, :-1]], 2)

    def place(x, fill):
        out = torch.full((B, N + 1), fill, dtype=torch.int64, device=DEV)
        return out.scatter_(1, at, x.to(torch.int64).reshape(B, -1))[:, :N]

    token, parent = place(drafts, EOS), place(up, -1)
    depth = place(p.expand(B, r, length), 0)
    token[:, 0], parent[:, 0], depth[:, 0] = first, -1, 0
    nodes = (1 + fresh.sum((1, 2))).to(torch.int32)
    # ancestors: every node's own draft names them
    words = -(-N // 64)
    see = torch.zeros(B, N + 1, words * 64, dtype=torch.bool, device=DEV)
    line = torch.where((p <= p[:, None]) & (node < N)[:, :, None, :], node[:, :, None, :],
                       words * 64).to(torch.int64)                       # [B, r, p, ancestor]
    one = torch.zeros(B, r * length, words * 64 + 1, dtype=torch.bool, device=DEV)
    one.scatter_(2, line.view(B, r * length, length), True)
    see.scatter_(1, at[:, :, None].expand(-1, -1, words * 64), one[:, :, :words * 64])
    see = see[:, :N]
    see[:, 0] = False
    see[:, 0, 0] = True
    bits = see.view(B, N, words, 64).to(torch.int64) << torch.arange(64, device=DEV)
    return (token.to(torch.int32), parent.to(torch.int32), depth.to(torch.int32), bits.sum(3),
            nodes)


def _plain_write(s):
    page = s["case"]["page"]
    at, off = s["slots"] // page, s["slots"] % page
    for name in ("k", "v"):
        x = s[name].to(torch.float32)
        pages = s[name + "_pages"]
        if s[name + "_exp"] is not None:
            e = _exponents(x)
            s[name + "_exp"][at, :, off] = (e + 127).to(torch.uint8)
            x = x * _power(-e)[..., None]
            pages.view(torch.uint8)[at, :, off] = x.to(pages.dtype).view(torch.uint8)
        else:
            pages[at, :, off] = x.to(pages.dtype)
    return s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"]


def _values(pages, exp, at, off, dtype=torch.float32):
    if exp is None:
        return pages[at, :, off].to(dtype)
    x = pages.view(torch.uint8)[at, :, off].view(pages.dtype).to(dtype)
    return x * _power(exp[at, :, off].to(torch.int32) - 127)[..., None].to(dtype)


def _plain_read(s):
    page, dtype = s["case"]["page"], DT[s["case"]["dtype"]]
    at, off = s["slots"] // page, s["slots"] % page
    return (_values(s["k_pages"], s["k_exp"], at, off).to(dtype),
            _values(s["v_pages"], s["v_exp"], at, off).to(dtype))


def _plain_attend(s):
    case = s["case"]
    B, hk, G, D, page = case["B"], case["heads"], case["group"], case["dim"], case["page"]
    H, L, n = hk * G, s["longest"], s["most"]
    pos = torch.arange(L, device=DEV)
    at = s["table"][:, pos // page].to(torch.int64)                      # [B, L]
    off = (pos % page).expand(B, L)
    k = _values(s["k_pages"], s["k_exp"], at, off).permute(0, 2, 3, 1).contiguous()
    starts = s["rows"].to(torch.int64)
    ns = starts[1:] - starts[:-1]
    t = torch.arange(n, device=DEV)
    row = (starts[:-1, None] + t).clamp(max=int(s["q"].numel() // (H * D)) - 1)
    q = s["q"].reshape(-1, H, D)[row].to(torch.float32)                  # [B, n, H, D]
    q = q.view(B, n, hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, hk, n * G, D)
    sc = torch.matmul(q, k).mul_(1.0 / math.sqrt(D)).view(B, hk, n, G, L)
    del k
    before = s["lengths"].to(torch.int64) - ns                           # cached before the chunk
    j = pos - before[:, None]                                            # [B, L]: chunk token
    see = (j[:, None] <= t[:, None]) if s["mask"] is None else (j < 0)[:, None] | _bits(s, j, n)
    see = see & (pos < s["lengths"][:, None])[:, None]                   # [B, n, L]
    sc.masked_fill_(~see[:, None, :, None], -math.inf)
    m = sc.amax(-1, keepdim=True).clamp(min=-3e38)
    sc.sub_(m).exp_()
    total = sc.sum(-1, keepdim=True)
    v = _values(s["v_pages"], s["v_exp"], at, off).transpose(1, 2).contiguous()
    out = torch.matmul(sc.view(B, hk, n * G, L), v).view(B, hk, n, G, D)
    out = (out / total.clamp(min=1e-37)).permute(0, 2, 1, 3, 4).reshape(B, n, H, D)
    lse = (m + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, n, H)
    if s["starts"] is not None:
        T = s["q"].shape[0]
        i = torch.arange(T, device=DEV)
        b = torch.searchsorted(starts[1:], i, right=True)
        out, lse = out[b, i - starts[b]], lse[b, i - starts[b]]
    out = out.to(DT[case["dtype"]])
    return (out, lse) if case["lse"] else out


def _bits(s, j, n):
    """[B, n, L]: whether chunk row t sees chunk token j."""
    words = s["mask"].view(j.shape[0], n, -1)
    c = j.clamp(min=0, max=words.shape[2] * 64 - 1)
    w = words.gather(2, (c // 64)[:, None].expand(-1, n, -1))
    return ((w >> (c % 64)[:, None]) & 1).to(torch.bool) & (j >= 0)[:, None]


def _plain_accept(s):
    case = s["case"]
    B, N, V, most = case["B"], case["N"], case["V"], case["length"]
    x = s["logits"]
    best = x.amax(-1, keepdim=True)
    g = torch.where(x == best, torch.arange(V, device=DEV, dtype=torch.int32), V).amin(-1)
    up = s["parent"].to(torch.int64).clamp(min=0)
    u = torch.arange(N, device=DEV)
    good = (s["token"] == g.gather(1, up)) | (u == 0)
    sees = ((s["mask"][:, :, None, :] >> torch.arange(64, device=DEV)[:, None]) & 1).transpose(
        2, 3).reshape(B, N, -1)[:, :, :N].to(torch.bool)
    on = (~sees | good[:, None]).all(2) & (u < s["nodes"][:, None])
    order = torch.where(on, u, N).sort(1)[0][:, :most]
    path = torch.where(order < N, order, -1).to(torch.int32)
    if N < most:
        path = torch.cat([path, torch.full((B, most - N), -1, dtype=torch.int32, device=DEV)], 1)
    length = (path >= 0).sum(1)
    last = path.gather(1, (length - 1).clamp(min=0)[:, None]).to(torch.int64).clamp(min=0)
    return path, length.to(torch.int32), g.gather(1, last)[:, 0]


_PLAIN = {"tree": lambda s: _plain_tree(s["drafts"], s["count"], s["first"], s["case"]["N"]),
          "write": _plain_write, "read": _plain_read, "attend": _plain_attend,
          "accept": _plain_accept}


# ---- what a pass cannot do without ----------------------------------------------------------


def work(case):
    kind = case["kind"]
    B = case.get("B", 0)
    if kind == "tree":
        N, words = case["N"], -(-case["N"] // 64)
        return {"bytes": 4 * B * (case["r"] * case["length"] + 3) + B * N * (12 + 8 * words),
                "flops": 0}
    if kind == "accept":
        # the logits of the accepted paths' nodes alone
        return {"bytes": sum(_accepted(case)) * case["V"] * SIZE[case["dtype"]]
                + 4 * B * (2 * case["N"] + case["length"] + 3), "flops": 0}
    heads, dim, es = case["heads"], case["dim"], SIZE[case["cache"]]
    row = heads * (dim * es + (case["cache"] == "f8"))
    if kind in ("write", "read"):
        return {"bytes": case["n"] * (2 * (row + heads * dim * SIZE[case["dtype"]]) + 8),
                "flops": 0}
    lengths, ns = _lengths(case, 0)
    H, page = heads * case["group"], case["page"]
    # visible pairs: the whole context, and of a chunk the earlier half (of a tree a few nodes)
    pairs = sum(n * (l - n) + (n * 5 if case["tree"] else n * (n + 1) // 2)
                for l, n in zip(lengths, ns))
    T = sum(ns)
    return {"bytes": 2 * sum(lengths) * row + 2 * T * H * dim * SIZE[case["dtype"]]
            + 4 * sum(-(-x // page) for x in lengths) + (4 * T * H if case["lse"] else 0)
            + (8 * T * -(-case["n"] // 64) if case["tree"] else 0),
            "flops": 4 * pairs * H * dim}


# ---- 64 bits --------------------------------------------------------------------------------


def exact(case, seed):
    kind = case["kind"]
    if kind in ("tree", "accept"):
        return None
    s = _inputs(case, seed)
    page, f64 = case["page"], torch.float64
    if kind == "read":
        out = []
        for name in ("k", "v"):
            x, e = s[name + "_pages"].transpose(1, 2).flatten(0, 1), s[name + "_exp"]
            x = x.view(torch.uint8)[s["slots"]].view(x.dtype) if e is not None else x[s["slots"]]
            x = x.to(f64)
            if e is not None:
                x = x * torch.exp2(e.transpose(1, 2).flatten(0, 1)[s["slots"]].to(f64)
                                   - 127.0)[..., None]
            out.append(x)
        return tuple(out)
    if kind == "write":
        out = []
        for name in ("k", "v"):
            x, e = s[name].to(f64), s[name + "_exp"]
            pages = s[name + "_pages"].to(f64)
            if e is not None:
                # the power of two at which the largest value lies in (224, 448]
                top = x.abs().amax(2).clamp(min=2.0 ** -117)
                b = torch.ceil(torch.log2(top / 448.0)).clamp(min=-126.0)
                y = x * torch.exp2(-b)[..., None]
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                x = torch.round(y / step) * step
            flat = pages.transpose(1, 2).flatten(0, 1)
            flat[s["slots"]] = x
            out.append(flat.view(-1, page, case["heads"], case["dim"]).transpose(1, 2))
        return tuple(out) + (None, None)
    hk, G, D = case["heads"], case["group"], case["dim"]
    H = hk * G
    lengths, ns = _lengths(case, seed)
    q = s["q"].reshape(-1, H, D)
    outs, lses, a = [], [], 0
    for b, (L, n) in enumerate(zip(lengths, ns)):
        pos = torch.arange(L, device=DEV)
        slot = s["table"][b, pos // page].to(torch.int64) * page + pos % page
        kv = []
        for name in ("k", "v"):
            x, e = s[name + "_pages"], s[name + "_exp"]
            x = x.transpose(1, 2).reshape(-1, hk, D) if e is None else x.view(
                torch.uint8).transpose(1, 2).reshape(-1, hk, D)
            x = x[slot] if e is None else x[slot].view(DT["f8"])
            x = x.to(f64)
            if e is not None:
                x = x * torch.exp2(e.transpose(1, 2).reshape(-1, hk)[slot].to(f64) - 127)[..., None]
            kv.append(x)
        see = torch.ones(n, L, dtype=torch.bool, device=DEV)
        if s["mask"] is None:
            see[:, L - n:] = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
        else:
            w = s["mask"].view(case["B"], n, -1)[b]
            i = torch.arange(n, device=DEV)
            see[:, L - n:] = ((w[:, i // 64] >> (i % 64)) & 1) == 1
        o, z = [], []
        for h in range(H):
            sc = q[a:a + n, h].to(f64) @ kv[0][:, h // G].t().contiguous() / math.sqrt(D)
            sc = sc.masked_fill(~see, -math.inf)
            z.append(torch.logsumexp(sc, 1))
            o.append(torch.exp(sc - z[-1][:, None]) @ kv[1][:, h // G].contiguous())
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(z, 1))
        a += n
    out, lse = torch.cat(outs), torch.cat(lses)
    if s["starts"] is None:
        out, lse = out.view(s["q"].shape), lse.view(s["q"].shape[:3])
    return (out, lse) if case["lse"] else out
