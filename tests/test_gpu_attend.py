"""Attention of chunks over a paged cache on the GPU against the plain oracle in 64 bits.

Tolerance of an element, from the arithmetic (u = half a step of the type, eps / 2):
 * the output is rounded once: u |out|;
 * each weight is rounded once to the type: u sum_p w_p |v_p| =: u mag;
 * a score is an fp32 sum of dim exact products and some factors: it is off by at most
   (dim + 4) 2^-24 |scale| sum |q_d k_d|, a weight relative to the sum by twice that;
 * exponentials and the rescaling of the running sums: 2^-20, and 2 L 2^-24 for fp32 sums over
   L keys;
 * f16: below its normal numbers an output is off by 2^-25, and a weight (kept at 2^10 times its
   value against the row's largest) by 2^-35 of the largest |v|, for each key.
None of these was taken from a run."""
import numpy as np
import pytest
import torch

from oracle import verify as ov

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}


def say(*a):
    print(*a, flush=True)


class Case:
    """Sequences of ctx[b] cached and ns[b] new tokens in a cache whose unused places hold NaN."""

    def __init__(self, seed, ctx, ns, heads, group, dim, page, dtype, cache, mask=None,
                 ragged=False, gap=0, sink=False):
        rng = self.rng = np.random.default_rng(seed)
        self.ctx, self.ns, self.B = ctx, ns, len(ctx)
        self.heads, self.H, self.dim, self.page = heads, heads * group, dim, page
        self.dtype, self.cache, self.ragged = dtype, cache, ragged
        self.lens = [c + n for c, n in zip(ctx, ns)]
        used = [-(-max(0, l) // page) for l in self.lens]
        pages = sum(used) + 2
        self.width = max(1, max(used)) + 1
        order = rng.permutation(pages)
        self.table = rng.choice([-1, pages, 1 << 30, -(1 << 31)], (self.B, self.width)).astype(
            np.int32)
        a = 0
        for b, u in enumerate(used):
            self.table[b, :u] = order[a:a + u]
            a += u
        shape = (pages, heads, page, dim)
        self.bits, self.exp, self.val = {}, {}, {}
        for name in "kv":
            x = rng.standard_normal(shape) * np.exp(rng.normal(0, 0.5, (heads, 1, dim)))
            x *= np.exp(rng.normal(0, 0.5, (pages, heads, page, 1)))
            if sink and name == "v":               # values of some tokens far below the others'
                x[:, :, ::3] *= 2.0 ** -30
                x[:, :, 1::7] = 0.0
            if cache == "f8":
                c, e = ov.quantise(x)
                v = ov.dequantise(c, e)
            else:
                t = torch.from_numpy(x).to(torch.float32).to(DT[cache])
                c, e, v = t.view(torch.int16).numpy().copy(), None, t.to(torch.float64).numpy()
            self.bits[name], self.exp[name], self.val[name] = c, e, v
        live = np.zeros((pages, page), bool)
        for b, l in enumerate(self.lens):
            for p in range(max(0, l)):
                live[self.table[b, p // page], p % page] = True
        for name in "kv":                          # what nobody may see
            bad = {"f8": 0x7f, "f16": 0x7e00 if name == "k" else 0x7c00,
                   "bf16": 0x7fc0 if name == "k" else 0x7f80}[cache]
            self.bits[name][np.broadcast_to(~live[:, None, :, None], shape)] = bad
            if cache == "f8":
                self.exp[name][np.broadcast_to(~live[:, None], shape[:3])] = 255
        self.starts = np.concatenate([[gap], gap + np.cumsum(ns)]).astype(np.int32)
        self.T = int(self.starts[-1]) + gap
        q = rng.standard_normal((self.T, self.H, dim)) * np.exp(rng.normal(0, 0.3, (1, self.H, dim)))
        self.q = torch.from_numpy(q).to(torch.float32).to(DT[dtype])
        n = max(ns)
        self.mask = None
        if mask is not None:
            W = -(-n // 64)
            self.mask = rng.integers(0, 1 << 63, (self.T, W), dtype=np.uint64) * np.uint64(2) | \
                rng.integers(0, 2, (self.T, W), dtype=np.uint64)
            if mask == "sparse":
                self.mask &= rng.integers(0, 1 << 63, (self.T, W), dtype=np.uint64)
                self.mask[::3] = 0
            if mask == "tree":
                self.mask[:] = 0
                for b in range(self.B):
                    anc = [set()]
                    for t in range(ns[b]):
                        s = {t} | (anc[int(rng.integers(0, len(anc)))])
                        anc.append(s)
                        for j in s:
                            self.mask[self.starts[b] + t, j // 64] |= np.uint64(1) << np.uint64(
                                j % 64)

    def see(self, b):
        n, L = self.ns[b], max(0, self.lens[b])
        s = np.ones((n, L), bool)
        j = np.arange(L) - self.ctx[b]
        if self.mask is None:
            return j[None] <= np.arange(n)[:, None]
        for i in range(L):
            if j[i] >= 0:
                w = self.mask[self.starts[b]:self.starts[b + 1], j[i] // 64]
                s[:, i] = (w >> np.uint64(j[i] % 64)) & np.uint64(1)
        return s

    def tensors(self):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        kp, vp = (t(self.bits[n]).view(DT[self.cache]) for n in "kv")
        ke, ve = (t(self.exp[n]) if self.cache == "f8" else None for n in "kv")
        kw = dict(k_exp=ke, v_exp=ve)
        # queries as a slice of a wider projection
        wide = torch.full((self.T, self.H + 3, self.dim), float("nan"), dtype=DT[self.dtype])
        wide[:, 1:1 + self.H] = self.q
        q = wide.to(DEV)[:, 1:1 + self.H]
        mask = t(self.mask.view(np.int64)) if self.mask is not None else None
        if self.ragged:
            kw["starts"] = t(self.starts)
        else:
            q = q.unflatten(0, (self.B, self.ns[0]))
            mask = mask.unflatten(0, (self.B, self.ns[0])) if mask is not None else None
        lens = np.array(self.lens, np.int32)
        return (q, kp, vp, t(self.table), t(lens)), dict(kw, mask=mask)

    def check(self, scale=None, **more):
        from paper_2502_15572_amd import paged_attention
        args, kw = self.tensors()
        out = torch.full(args[0].shape, 7.0, dtype=DT[self.dtype], device=DEV)
        lse = torch.full(args[0].shape[:-1], 7.0, device=DEV)
        paged_attention(*args, **kw, scale=scale, with_lse=True, out=(out, lse), **more)
        torch.cuda.synchronize()
        self.compare(out, lse, scale)
        alone = paged_attention(*args, **kw, scale=scale)
        a, b = self.starts[0], self.starts[-1]
        assert torch.equal(alone.view(-1, self.H, self.dim)[a:b], out.view(
            -1, self.H, self.dim)[a:b])
        return out, lse

    def compare(self, out, lse, scale=None):
        out = out.reshape(self.T, self.H, self.dim).to(torch.float64).cpu().numpy()
        lse = lse.reshape(self.T, self.H).to(torch.float64).cpu().numpy()
        scale = self.dim ** -0.5 if scale is None else scale
        u = torch.finfo(DT[self.dtype]).eps / 2
        q = self.q.to(torch.float64).numpy()
        worst = 0.0
        for b in range(self.B):
            L = max(0, self.lens[b])
            p = np.arange(L)
            k, v = (self.val[n].transpose(0, 2, 1, 3)[self.table[b, p // self.page], p % self.page]
                    for n in "kv")
            r = slice(self.starts[b], self.starts[b + 1])
            want, wl, mag, size = ov.attend(q[r], k, v, self.see(b), scale)
            ds = (self.dim + 4) * 2.0 ** -24 * size
            rel = 2.2 * ds + 2.0 ** -20 + (2 * L + 64) * 2.0 ** -24
            tol = u * np.abs(want) + (u + rel)[..., None] * mag + 1e-38
            if self.dtype == "f16":
                top = np.abs(v).max() if L else 0.0
                tol = tol + 2.0 ** -25 + L * 2.0 ** -35 * top
            err = np.abs(out[r] - want)
            assert np.isfinite(out[r]).all(), "sequence %d" % b
            worst = max(worst, float((err / tol).max()) if err.size else 0.0)
            assert (err <= tol).all(), ("sequence %d" % b, float((err / tol).max()))
            none = np.isneginf(wl)
            assert (np.isneginf(lse[r]) == none).all()
            tl = ds + 2.0 ** -20 + (L + 8) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(none, 0, wl))
            assert (np.abs(lse[r][~none] - wl[~none]) <= tl[~none]).all()
        say("worst error / tolerance %.3f" % worst)
        # rows of no chunk are left as they were
        for r in (slice(0, self.starts[0]), slice(self.starts[-1], self.T)):
            assert (out[r] == 7).all() and (lse[r] == 7).all()


STEP = [  # ctx, heads, group, dim, page, dtype, cache: one new token of each sequence
    ([0], 1, 1, 64, 16, "bf16", "bf16"), ([0, 1, 15, 16, 17, 63, 64], 2, 4, 128, 16, "f16", "f16"),
    ([300, 1, 129], 3, 2, 128, 32, "bf16", "f8"), ([511, 40], 2, 8, 64, 64, "f16", "f8"),
    ([1000], 1, 16, 80, 8, "bf16", "bf16"), ([700, 3], 2, 1, 256, 16, "bf16", "bf16"),
    ([257], 1, 7, 96, 1, "f16", "f16"), ([90, 200], 4, 3, 8, 4, "bf16", "bf16"),
    ([333], 2, 5, 136, 128, "f16", "f8"), ([5000, 17], 2, 4, 128, 16, "bf16", "bf16"),
    ([20001], 1, 8, 128, 64, "bf16", "f8"), ([9000], 2, 2, 256, 32, "f16", "f8"),
    ([130] * 40, 2, 2, 72, 16, "bf16", "f8"), ([64], 1, 71, 64, 16, "f16", "f16"),
    ([100, 260], 1, 32, 128, 16, "bf16", "bf16"), ([77], 2, 40, 248, 2, "bf16", "f8")]


@pytest.mark.parametrize("ctx,heads,group,dim,page,dtype,cache", STEP, ids=str)
def test_one_token(gpu_lib, ctx, heads, group, dim, page, dtype, cache):
    say("attend step", ctx[:8], heads, group, dim, page, dtype, cache)
    Case(len(ctx) + dim, ctx, [1] * len(ctx), heads, group, dim, page, dtype, cache).check()


CHUNK = [  # ctx, n, heads, group, dim, page, dtype, cache, mask
    ([0, 100], 7, 2, 2, 64, 16, "bf16", "bf16", None), ([33], 91, 2, 1, 128, 16, "f16", "f16", "tree"),
    ([200, 1], 64, 1, 4, 128, 32, "bf16", "f8", "tree"), ([0, 5], 65, 2, 2, 128, 16, "bf16", "bf16",
                                                       "any"),
    ([0, 0, 9], 30, 3, 1, 64, 8, "f16", "f16", "sparse"), ([500], 130, 1, 2, 96, 64, "bf16", "bf16",
                                                         "sparse"),
    ([17], 200, 2, 4, 128, 16, "bf16", "bf16", None), ([1200], 48, 1, 8, 128, 16, "f16", "f8", None),
    ([40], 150, 1, 1, 256, 16, "f16", "f16", None), ([64], 129, 1, 3, 80, 32, "bf16", "f8", "any"),
    ([3000], 16, 2, 4, 64, 128, "bf16", "bf16", "tree"), ([10], 20, 2, 2, 256, 4, "bf16", "f8", "tree"),
    ([2047], 33, 1, 1, 128, 256, "f16", "f16", None)]


@pytest.mark.parametrize("ctx,n,heads,group,dim,page,dtype,cache,mask", CHUNK, ids=str)
def test_chunk(gpu_lib, ctx, n, heads, group, dim, page, dtype, cache, mask):
    say("attend chunk", ctx, n, heads, group, dim, page, dtype, cache, mask)
    Case(n + dim, ctx, [n] * len(ctx), heads, group, dim, page, dtype, cache, mask).check()


RAGGED = [  # ctx, ns, heads, group, dim, page, dtype, cache, mask, gap
    ([0, 50, 7], [1, 0, 40], 2, 2, 64, 16, "bf16", "bf16", None, 0),
    ([300, 0, 1, 65], [2, 130, 1, 0], 2, 4, 128, 16, "f16", "f16", None, 3),
    ([129, 40], [17, 64], 1, 5, 80, 32, "bf16", "f8", "any", 2),
    ([10] * 70, list(range(70)), 1, 2, 64, 8, "bf16", "bf16", None, 1),
    ([600, 20, 5], [1, 300, 70], 2, 4, 128, 64, "bf16", "f8", None, 5),
    ([0, 200, 0], [90, 0, 128], 1, 1, 256, 16, "f16", "f16", "sparse", 0),
    ([0], [0], 2, 2, 64, 16, "bf16", "bf16", None, 4)]


@pytest.mark.parametrize("ctx,ns,heads,group,dim,page,dtype,cache,mask,gap", RAGGED, ids=str)
def test_ragged(gpu_lib, ctx, ns, heads, group, dim, page, dtype, cache, mask, gap):
    say("attend ragged", ctx[:6], ns[:6], heads, group, dim, page, dtype, cache, mask, gap)
    Case(sum(ns) + dim, ctx, ns, heads, group, dim, page, dtype, cache, mask, ragged=True,
         gap=gap).check()


def test_lengths_below_the_chunk(gpu_lib):
    """Sequences with fewer tokens than their chunk has rows: the first rows have no position."""
    say("attend: short lengths")
    Case(3, [-5, -9, -20, -1], [9, 9, 9, 9], 2, 2, 64, 16, "bf16", "bf16").check()
    Case(4, [-70, -150], [150, 150], 1, 2, 128, 16, "f16", "f16").check()


@pytest.mark.parametrize("dtype,cache", [("f16", "f8"), ("bf16", "f8"), ("f16", "f16")])
def test_values_of_very_different_size(gpu_lib, dtype, cache):
    """Tokens whose values are 2^-30 of the others' or zero, seen with large and small weights."""
    say("attend: sinks", dtype, cache)
    for n, ctx in ((1, 700), (70, 90)):
        Case(n, [ctx], [n], 2, 2, 128, 16, dtype, cache, sink=True).check()


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(gpu_lib, scale):
    say("attend: scale", scale)
    for n in (1, 80):
        Case(5, [150, 0], [n, n], 2, 3, 64, 16, "bf16", "bf16").check(scale=scale)


@pytest.mark.parametrize("n,ctx", [(1, 200), (20, 100), (140, 64)])
@pytest.mark.parametrize("cache", ["f16", "f8"])
def test_nan_and_infinity_in_masked_places(gpu_lib, n, ctx, cache):
    """Chunk tokens that some rows see hold NaN and infinities: the rows that do not see them
    are as if they were not there, the rows that do are not finite."""
    from paper_2502_15572_amd import paged_attention
    say("attend: masked NaN", n, ctx, cache)
    c = Case(n + ctx, [ctx], [n], 2, 2, 64, 16, "f16", cache, mask="any")
    bad = sorted({0, n // 2, n - 1})
    for j in bad:
        c.mask[:, j // 64] &= ~(np.uint64(1) << np.uint64(j % 64))
    for t in range(0, n, 3):
        c.mask[t, bad[0] // 64] |= np.uint64(1) << np.uint64(bad[0] % 64)
    for j in bad:
        pg, o = c.table[0, (ctx + j) // 16], (ctx + j) % 16
        for name in "kv":
            c.bits[name][pg, :, o] = 0x7f if cache == "f8" else (0x7c00 if name == "v" else 0x7e00)
    args, kw = c.tensors()
    out, lse = paged_attention(*args, **kw, with_lse=True)
    out = out.view(n, c.H, 64)
    sees = np.zeros(n, bool)
    sees[::3] = True
    assert not torch.isfinite(out[torch.from_numpy(sees)]).any()
    for name in "kv":                       # the oracle without them
        for j in bad:
            pg, o = c.table[0, (ctx + j) // 16], (ctx + j) % 16
            c.val[name][pg, :, o] = 0.0
    full = c.see(0)
    want, wl, mag, size = ov.attend(
        c.q.to(torch.float64).numpy(), *(c.val[m].transpose(0, 2, 1, 3)[
            c.table[0, np.arange(ctx + n) // 16], np.arange(ctx + n) % 16] for m in "kv"), full,
        64 ** -0.5)
    got = out.to(torch.float64).cpu().numpy()[~sees]
    u = 2.0 ** -11
    rel = 2.2 * 68 * 2.0 ** -24 * size + 2.0 ** -20 + (2 * (ctx + n) + 64) * 2.0 ** -24
    tol = u * np.abs(want) + (u + rel)[..., None] * mag + 2.0 ** -25 + (ctx + n) * 2.0 ** -35 * 1e3
    assert (np.abs(got - want[~sees]) <= tol[~sees]).all()


def test_far_positions(gpu_lib):
    """Byte offsets past 2^32 in the cache and a long table: the last pages of a cache of 2^33
    bytes are read."""
    from paper_2502_15572_amd import paged_attention
    say("attend: far pages")
    pages, heads, page, dim = 16400, 4, 256, 128           # 4.3 GB each of keys and values
    kp = torch.zeros(pages, heads, page, dim, dtype=torch.float16, device=DEV)
    vp = torch.zeros_like(kp)
    g = torch.Generator(device=DEV).manual_seed(1)
    last = torch.randn(2, heads, 2 * page, dim, device=DEV, generator=g).to(torch.float16)
    for t, x in ((kp, last[0]), (vp, last[1])):
        t[-2:] = x.view(heads, 2, page, dim).transpose(0, 1)
    table = torch.tensor([[pages - 2, pages - 1]], dtype=torch.int32, device=DEV)
    q = torch.randn(1, 1, heads, dim, device=DEV, generator=g).to(torch.float16)
    n = torch.tensor([2 * page - 3], dtype=torch.int32, device=DEV)
    out = paged_attention(q, kp, vp, table, n)
    k, v = (x[:, :2 * page - 3].to(torch.float64) for x in last)
    w = torch.softmax((k * q[0, 0].to(torch.float64)[:, None]).sum(-1) * dim ** -0.5, 1)
    want = (w[:, :, None] * v).sum(1)
    assert float((out[0, 0].to(torch.float64) - want).abs().max()) < 2e-3 * float(v.abs().max())


@pytest.mark.parametrize("n", [1, 40, 200])
def test_replayed_graphs_beside_each_other(gpu_lib, n):
    """Two calls captured on one stream, replayed on two streams at once beside eager calls; and
    other lengths and pages put in place between replays."""
    from paper_2502_15572_amd import paged_attention
    say("attend: graphs", n)
    cases = [Case(s, [700, 90], [n, n], 2, 4, 128, 16, "bf16", "bf16") for s in (1, 2)]
    given = [c.tensors() for c in cases]
    want = [paged_attention(*a, **k) for a, k in given]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graphs = []
    for a, k in given:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = paged_attention(*a, **k, stream=s)
        graphs.append((g, out))
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for g, out in graphs:
            out.zero_()
        torch.cuda.synchronize()
        for (g, out), side in zip(graphs, sides):
            with torch.cuda.stream(side):
                g.replay()
        eager = [paged_attention(*a, **k) for a, k in given]
        torch.cuda.synchronize()
        for (g, out), w, e in zip(graphs, want, eager):
            assert torch.equal(out, w) and torch.equal(e, w)
    lens = given[0][0][4]
    lens -= 37                                             # shorter sequences, the same graph
    w = paged_attention(*given[0][0], **given[0][1])
    graphs[0][0].replay()
    torch.cuda.synchronize()
    assert torch.equal(graphs[0][1], w) and not torch.equal(w, want[0])


def test_streams_and_repeats(gpu_lib):
    """The same call on other streams and again gives the same bits."""
    from paper_2502_15572_amd import paged_attention
    say("attend: streams")
    c = Case(9, [900, 30, 4], [3, 3, 3], 2, 4, 128, 16, "f16", "f8")
    args, kw = c.tensors()
    want = paged_attention(*args, **kw)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [paged_attention(*args, **kw, stream=s) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("n", [1, 12, 150])
@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("bf16", "f8")])
def test_shared_pages(gpu_lib, n, dtype, cache):
    """Sequences with the same first pages, and a page twice in one table, give what copies of the
    pages give."""
    from paper_2502_15572_amd import paged_attention
    say("attend: shared pages", n, dtype, cache)
    c = Case(5, [640 - n, 640 - n], [n, n], 2, 2, 128, 64, dtype, cache)
    (q, kp, vp, table, lens), kw = c.tensors()
    q[1] = q[0]
    shared = table.clone()
    shared[1, :8] = shared[0, :8]                          # then pages of its own
    shared[:, 3] = shared[:, 1]
    args, ex = [kp.clone(), vp.clone()], {}
    for x in args:
        y = x.view(torch.uint8)
        for b in (0, 1):
            y[table[b, :10].long()] = y[shared[b, :10].long()].clone()
    for name in ("k_exp", "v_exp"):
        ex[name] = kw[name]
        if kw[name] is not None:
            ex[name] = kw[name].clone()
            for b in (0, 1):
                ex[name][table[b, :10].long()] = kw[name][shared[b, :10].long()].clone()
    got = paged_attention(q, kp, vp, shared, lens, **kw)
    want = paged_attention(q, *args, table, lens, mask=None, **ex)
    assert torch.equal(got, want) and torch.isfinite(got).all()


def test_chunks_that_do_not_ascend(gpu_lib):
    """Chunks that overlap, go back or leave the rows: nothing outside the rows is written."""
    from paper_2502_15572_amd import paged_attention
    say("attend: odd chunks")
    c = Case(6, [200] * 5, [7] * 5, 2, 4, 64, 16, "bf16", "bf16", ragged=True)
    (q, kp, vp, table, lens), kw = c.tensors()
    for starts in ([0, 35, 0, 35, 0, 35], [35, 20, 10, 5, 2, 0], [-5, 3, 50, 1 << 30, 7, 9],
                   [0, 0, 0, 0, 0, 1 << 30]):
        kw["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        buf = torch.full((35 + 64, c.H, c.dim), 7.0, dtype=torch.bfloat16, device=DEV)
        paged_attention(q, kp, vp, table, lens, **kw, out=buf[32:67])
        torch.cuda.synchronize()
        assert (buf[:32] == 7).all() and (buf[67:] == 7).all()


def test_more_blocks_than_a_launch_takes(gpu_lib):
    import ctypes
    from paper_2502_15572_amd import _lib
    say("attend: too many blocks")
    need = ctypes.c_int64()
    c = _lib.KvCache(None, None, None, None, 4, 16, 16, 64, _lib.F16)
    ask = lambda B: gpu_lib.dresd_paged_attention_workspace(c, 16, 0, 1, B, B, 5,  # noqa: E731
                                                            ctypes.byref(need))
    assert ask((1 << 20) - 1) == _lib.OK and need.value == 0
    assert ask(1 << 20) == _lib.EINVAL
    assert "blocks" in gpu_lib.dresd_last_error().decode()


@pytest.mark.parametrize("dtype,cache", [("bf16", "f8"), ("f16", "f8"), ("f16", "f16")])
@pytest.mark.parametrize("n,dim", [(32, 256), (33, 64), (64, 256), (65, 256), (64, 128), (65, 128),
                                   (97, 256), (130, 256)])
def test_where_kernels_meet(gpu_lib, n, dim, dtype, cache):
    """Numbers of rows on either side of what the launch plan goes by."""
    say("attend rows", n, dim, dtype, cache)
    Case(n + dim, [333, 20], [n, n], 2, 1, dim, 16, dtype, cache, "tree").check()


@pytest.mark.parametrize("n,words", [(70, 1), (5, 3), (1, 1), (130, 2), (64, 2)])
@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("bf16", "f8")])
def test_mask_words(gpu_lib, n, words, dtype, cache):
    """More words than the chunk has bits (whose further ones are set), and fewer."""
    say("attend: mask words", n, words, dtype, cache)
    c = Case(n + words, [90, 0], [n, n], 2, 2, 64, 16, dtype, cache, "any")
    full = np.full((c.T, max(words, c.mask.shape[1])), ~np.uint64(0))
    full[:, :c.mask.shape[1]] = c.mask
    if words < c.mask.shape[1]:
        full[:, words:] = 0
    c.mask = full                                          # what the oracle looks at
    (q, kp, vp, table, lens), kw = c.tensors()
    kw["mask"] = kw["mask"][..., :words].contiguous()
    from paper_2502_15572_amd import paged_attention
    out, lse = paged_attention(q, kp, vp, table, lens, **kw, with_lse=True)
    c.compare(out, lse)


def test_a_page_of_65536_tokens(gpu_lib):
    say("attend: one large page")
    Case(3, [5000, 64], [3, 3], 1, 2, 64, 65536, "bf16", "bf16").check()
