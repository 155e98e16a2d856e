"""The operators of batch verification together, as a decoding program uses them: a small
language model (one attention layer, random weights) decodes greedily with drafts from its own
datastore.  At each step the drafts become a tree, its keys and values enter the paged cache,
its queries attend over context and ancestors, the logits decide, and the accepted entries are
moved to their final slots.  Every token is checked against the model in 64 bits on the CPU, on
the tokens before it; and one step is captured into a graph and replayed."""
import numpy as np
import pytest
import torch

from oracle import verify as ov

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V, WIDTH, HEADS, GROUP, DIM, PAGE = 300, 96, 2, 2, 64, 16
Q = HEADS * GROUP


def say(*a):
    print(*a, flush=True)


class Model:
    """logits = E (x + Wo attention(x)), x = E[token] + P[position]; keys, values and queries
    in 16 bits."""

    def __init__(self, seed, dtype):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)
        self.dtype = dtype
        self.emb, self.pos = r(V, WIDTH), 0.5 * r(256, WIDTH)
        self.wqkv = r(WIDTH, (Q + 2 * HEADS) * DIM) * WIDTH ** -0.5
        self.wo = 2.0 * r(Q * DIM, WIDTH) * (Q * DIM) ** -0.5
        self.out = r(WIDTH, V) * WIDTH ** -0.5
        self.on = [t.to(DEV) for t in (self.emb, self.pos, self.wqkv, self.wo, self.out)]

    def qkv(self, token, position):
        emb, pos, wqkv, _, _ = self.on
        x = emb[token.long()] + pos[position.long()]
        h = (x @ wqkv).to(self.dtype).unflatten(-1, (Q + 2 * HEADS, DIM))
        return x, h[..., :Q, :], h[..., Q:Q + HEADS, :], h[..., Q + HEADS:, :]

    def logits(self, x, att):
        _, _, _, wo, out = self.on
        return (x + att.flatten(-2).to(torch.float32) @ wo) @ out

    def exact(self, tokens, f8):
        """Logits after every token of a sequence, in 64 bits, with the cache's rounding."""
        n = len(tokens)
        x = (self.emb[tokens] + self.pos[:n]).double()
        h = (x @ self.wqkv.double()).to(torch.float32).to(self.dtype).double().view(n, -1, DIM)
        q, k, v = h[:, :Q].numpy(), h[:, Q:Q + HEADS].numpy(), h[:, Q + HEADS:].numpy()
        if f8:
            k, v = (ov.dequantise(*ov.quantise(t)) for t in (k, v))
        o = ov.attend(q, k, v, np.tril(np.ones((n, n), bool)), DIM ** -0.5)[0]
        x = x + torch.from_numpy(o).reshape(n, -1) @ self.wo.double()
        return x @ self.out.double(), x


class Cache:
    def __init__(self, dtype, B, f8):
        self.width = 160 // PAGE
        pages = B * self.width + 3
        kind = torch.float8_e4m3fn if f8 else dtype
        self.k = torch.zeros(pages, HEADS, PAGE, DIM, dtype=kind, device=DEV)
        for t in (self.k,):
            t.view(torch.uint8).fill_(0x7f)             # NaN (or near it) wherever nothing is
        self.v = self.k.clone()
        self.ke = torch.full(self.k.shape[:3], 255, dtype=torch.uint8, device=DEV) if f8 else None
        self.ve = self.ke.clone() if f8 else None
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(0))
        self.table = order[:B * self.width].view(B, self.width).to(torch.int32).to(DEV)

    def slots(self, position):
        """Slots of positions [B, n] (negative: none)."""
        p = position.clamp(min=0).long()
        s = self.table.gather(1, p // PAGE).long() * PAGE + p % PAGE
        return torch.where(position < 0, -1, s).flatten().contiguous()

    def pages(self):
        return self.k, self.v, self.ke, self.ve


def forward(m, c, token, parent, depth, mask, nodes, lens):
    """One forward over trees behind contexts of lens tokens; (x, logits)."""
    from paper_2502_15572_amd import kv_write, paged_attention
    B, N = token.shape
    x, q, k, v = m.qkv(token, lens[:, None] + depth)
    at = torch.arange(N, device=DEV)
    # past the last node nothing is written
    where = torch.where(at < nodes[:, None], lens[:, None] + at, -1)
    kv_write(k.flatten(0, 1), v.flatten(0, 1), c.slots(where), *c.pages())
    att = paged_attention(q, c.k, c.v, c.table, (lens + N).to(torch.int32), mask=mask, k_exp=c.ke,
                          v_exp=c.ve)
    return x, m.logits(x, att)


def prefill(m, c, prompts):
    """Prompts in two ragged chunks; (the model's next token, lengths)."""
    from paper_2502_15572_amd import kv_write, paged_attention
    B = len(prompts)
    done = torch.zeros(B, dtype=torch.int64)
    for part in (0.4, 1.0):
        upto = torch.tensor([int(np.ceil(part * len(p))) for p in prompts])
        ns = upto - done
        starts = torch.cat([torch.zeros(1, dtype=torch.int64), ns.cumsum(0)]).to(torch.int32)
        tok = torch.tensor([t for p, a, b in zip(prompts, done, upto) for t in p[a:b]])
        pos = torch.cat([torch.arange(a, b) for a, b in zip(done, upto)])
        seq = torch.repeat_interleave(torch.arange(B), ns)
        x, q, k, v = m.qkv(tok.to(DEV), pos.to(DEV))
        s = c.table[seq.to(DEV), (pos // PAGE).to(DEV)].long() * PAGE + (pos % PAGE).to(DEV)
        kv_write(k, v, s, *c.pages())
        att = paged_attention(q, c.k, c.v, c.table, upto.to(torch.int32).to(DEV),
                              starts=starts.to(DEV), k_exp=c.ke, v_exp=c.ve)
        done = upto
    lg = m.logits(x, att)[(starts[1:] - 1).to(DEV)]
    return lg.argmax(1).to(torch.int32), done.to(torch.int32).to(DEV)


def decode(m, c, prompts, total, drafter):
    """Greedy decoding; (tokens of each sequence after its prompt, forwards, last states)."""
    from paper_2502_15572_amd import accept_drafts, draft_tree, kv_read, kv_write
    nxt, lens = prefill(m, c, prompts)
    B = len(prompts)
    out, forwards = [[] for _ in prompts], 0
    state = None
    while min(len(o) for o in out) < total:
        d, count = drafter(state, nxt, out)
        token, parent, depth, mask, nodes = draft_tree(d, count, nxt, 40)
        x, lg = forward(m, c, token, parent, depth, mask, nodes, lens)
        path, n, new = accept_drafts(lg, token, parent, nodes, d.shape[2])
        forwards += 1
        # the accepted nodes' entries move to the positions after the context
        at = torch.arange(path.shape[1], device=DEV)
        src = torch.where(path >= 0, lens[:, None] + path, -1)
        dst = torch.where(path >= 0, lens[:, None] + at, -1)
        kv_write(*kv_read(c.slots(src), *c.pages()), c.slots(dst), *c.pages())
        for b in range(B):
            out[b] += token[b, path[b, :n[b]].long()].tolist()
        last = path.gather(1, (n - 1)[:, None].long()).long()
        state = x.gather(1, last[:, :, None].expand(-1, -1, WIDTH))[:, 0]
        nxt, lens = new, lens + n
    return out, forwards


def no_drafts(state, nxt, out):
    d = nxt[:, None, None].expand(-1, 1, 2).clone()
    d[:, :, 1] = 0
    return d.contiguous(), torch.ones_like(nxt)


@pytest.mark.parametrize("dtype,f8", [(torch.float16, False), (torch.bfloat16, True)], ids=str)
def test_decoding_with_drafts(gpu_lib, dtype, f8):
    from paper_2502_15572_amd import Index, pack_drafts
    say("decode with drafts", dtype, f8)
    m = Model(3, dtype)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(1, V, n).tolist() for n in (5, 23, 16)]
    total = 40
    plain, steps = decode(m, Cache(dtype, 3, f8), prompts, total, no_drafts)
    # the datastore: states of what was decoded -> the six tokens that followed
    keys, values = [], []
    for p, o in zip(prompts, plain):
        seq = torch.tensor(p + o)
        st = m.emb[seq] + m.pos[: len(seq)]
        for i in range(len(p) - 1, len(seq) - 7):
            keys.append(st[i] / st[i].norm())
            values.append(seq[i + 1:i + 7])
    ix = Index(torch.stack(keys).to(DEV), torch.stack(values).to(torch.int32).to(DEV))

    def drafter(state, nxt, out):
        if state is None:
            return no_drafts(state, nxt, out)
        q = state / state.norm(dim=1, keepdim=True)
        _, _, tok = ix.search(q.contiguous(), 12, next_tok=nxt)
        return pack_drafts(tok, 8, 6)

    drafted, fewer = decode(m, Cache(dtype, 3, f8), prompts, total, drafter)
    say("tokens %d, forwards without drafts %d, with %d" % (total, steps, fewer))
    assert fewer < 0.75 * steps
    # Each token is the model's own: its logit is the largest up to the rounding of the 16-bit
    # attention output (2^-8 relative, through Wo and the output matrix: a sum of 96 products of
    # unit variance, x of size about 2) and of the weights.
    worst = 0.0
    for p, o in list(zip(prompts, plain)) + list(zip(prompts, drafted)):
        lg, _ = m.exact(torch.tensor(p + o), f8)
        lg = lg[len(p) - 1:len(p) + len(o) - 1]
        worst = max(worst, float((lg.amax(1) - lg[torch.arange(len(o)), torch.tensor(o)]).max()))
    say("worst gap to the best logit %.4f" % worst)
    assert worst < 0.05
    ix.close()


def test_a_captured_step(gpu_lib):
    """Tree, write, attention and acceptance of one step in a graph, replayed with other drafts
    in place."""
    from paper_2502_15572_amd import accept_drafts, draft_tree
    say("captured step")
    dtype = torch.float16
    m = Model(5, dtype)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(1, V, n).tolist() for n in (7, 30)]
    c = Cache(dtype, 2, False)
    nxt, lens = prefill(m, c, prompts)

    def drafts(seed):
        r = np.random.default_rng(seed)
        d = r.integers(0, 5, (2, 9, 5)).astype(np.int32)
        d[:, :, 0] = nxt.cpu().numpy()[:, None]
        return torch.from_numpy(d).to(DEV), torch.tensor([9, 4], dtype=torch.int32, device=DEV)

    def step():
        token, parent, depth, mask, nodes = draft_tree(d, count, nxt, 33)
        _, lg = forward(m, c, token, parent, depth, mask, nodes, lens)
        return (lg, token, mask) + accept_drafts(lg, token, parent, nodes)

    d, count = drafts(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for seed in (0, 1, 2, 3):
        new = drafts(seed)
        d.copy_(new[0])
        count.copy_(new[1])
        want = [t.clone() for t in step()]
        for t in got:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
