"""Beam search as a program runs it: attention over the shared prompt by hidden states (EL-attention) and over each beam's own
continuation by paged keys and values, joined under one softmax; scores of the tokens, the best of all beams, forks.

A toy decoder of one attention layer on token embeddings.  Every score that the search sees is checked against ordinary
multi-head attention in fp64 over the whole history of the beam it belongs to."""
import numpy as np
import pytest

import oracle
from paper_2105_04779_amd import workloads as wl
from helpers import device_weights, record, to_device

pytestmark = pytest.mark.gpu

PAGE = 4


class Model:
    def __init__(self, dtype, heads, d_m, V, seed):
        from paper_2105_04779_amd import el_attn
        self.dtype, self.heads, self.d_m, self.d_k, self.V = dtype, heads, d_m, d_m // heads, V
        self.w = wl.custom("search", dtype=dtype, B=1, beam=1, heads=heads, d_m=d_m, d_k=self.d_k, n=8, index=90 + seed)
        self.W = wl.weights(self.w)
        self.W["bk"] = wl.round_to_storage(self.W["bk"] * np.float32(25), dtype)       # visible across the two key sets
        g = np.random.default_rng(seed)
        self.E = wl.round_to_storage(g.standard_normal((V, d_m), dtype=np.float32), dtype)
        self.Wd, self.Ed = device_weights(self.W, dtype), to_device(self.E, dtype)
        self.layer = lambda B, x, n: el_attn.ElAttention(self.Wd, heads=heads, d_k=self.d_k, dtype=dtype, max_batch=B * x, max_beam=x, max_n=n)

    def project(self, x, name):
        """x W + b of embedded tokens, heads apart, rounded to the storage type."""
        y = x.float() @ self.Wd["W" + name].float() + self.Wd["b" + name].float()
        return y.to(x.dtype).unflatten(-1, (self.heads, self.d_k))

    def logits(self, h):
        return h.float() @ self.Ed.float().t() / 8.0

    def exact(self, prompt, history):
        """Logits in fp64 of a beam that has the prompt's hidden states and its own tokens, the last of which asks."""
        x = self.E[history].astype(np.float64)
        H = np.concatenate([prompt.astype(np.float64), x])[None]
        out = oracle.mha_reference(H.astype(np.float32), np.array([H.shape[1]], np.int32), x[None, -1:].astype(np.float32), self.W["Wq"], self.W["bq"],
                                   self.W["Wk"], self.W["bk"], self.W["Wv"], self.W["bv"], self.W["Wo"], self.W["bo"],
                                   heads=self.heads, d_k=self.d_k)
        return out[0, 0] @ self.E.astype(np.float64).T / 8.0


class Pages:
    """Host side of the pages: who holds which, and which are free.  A page is shared until a beam has to write into it."""

    def __init__(self, pages, rows, columns):
        self.held, self.free, self.users = [[] for _ in range(rows)], list(range(pages)), [0] * pages
        self.columns = columns

    def take(self):
        p = self.free.pop()
        self.users[p] = 1
        return p

    def fork(self, parents):
        """Every row goes on from its parent; returns the (source, destination) pages to copy where two go on from one."""
        old, self.held = self.held, [list(self.held[p]) for p in parents]
        users, pairs = [0] * len(self.users), []
        for row in self.held:
            for p in row:
                users[p] += 1
        for p, (was, now) in enumerate(zip(self.users, users)):
            if was and not now:
                self.free.append(p)
        self.users = users
        return pairs

    def room(self, length):
        """Room for position length - 1 in every row: a page of its own to write into."""
        pairs = []
        for row in self.held:
            if len(row) * PAGE < length:
                row.append(self.take())
            elif self.users[row[-1]] > 1:
                self.users[row[-1]] -= 1
                pairs.append((row[-1], self.take()))
                row[-1] = pairs[-1][1]
        return pairs

    def table(self):
        import torch
        t = torch.full((len(self.held), self.columns), -1, dtype=torch.int32)
        for r, row in enumerate(self.held):
            t[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
        return t


@pytest.mark.parametrize("dtype,heads,d_m", [("bf16", 8, 512), ("f16", 16, 1024), ("f32", 4, 64)])
def test_search_over_a_prompt_and_paged_continuations(dtype, heads, d_m):
    import torch
    from paper_2105_04779_amd import el_attn
    B, x, n, V, steps = 3, 4, 60, 1013, 11
    model = Model(dtype, heads, d_m, V, seed=2)
    g = np.random.default_rng(1)
    lens = np.array([60, 33, 7], dtype=np.int32)
    H = wl.round_to_storage(g.standard_normal((B, n, d_m), dtype=np.float32), dtype)
    Hd, Ld = to_device(H, dtype), torch.from_numpy(lens).cuda()
    layer = model.layer(B, x, n)
    pool = torch.full((2, 64, PAGE, heads, d_m // heads), float("nan"), device="cuda", dtype=Hd.dtype)
    cache, pages = el_attn.PagedCache(pool[0], pool[1]), Pages(64, B * x, 4)
    tokens = torch.tensor([[7 + 3 * b] * x for b in range(B)])
    total = torch.full((B, x), -float("inf"))
    total[:, 0] = 0.0                                                # all beams start alike: only the first one's alternatives count
    history = [[int(t)] for t in tokens.reshape(-1)]
    forks = 0
    for step in range(steps):
        pairs = pages.room(step + 1)
        forks += len(pairs)
        if pairs:
            src, dst = torch.tensor(pairs, dtype=torch.int32).t().contiguous().cuda()
            counts = torch.full_like(src, step % PAGE)
            cache.copy_pages(src, dst, counts)
        table = pages.table().cuda()
        lengths = torch.full((B * x,), step + 1, dtype=torch.int32, device="cuda")
        h = model.Ed[tokens.reshape(-1).cuda()]                      # [B*x, d_m]
        cache.append(model.project(h, "k")[:, None], model.project(h, "v")[:, None], table, lengths)
        prompt = layer.decode_segment(Hd, Ld, h.view(B, x, d_m))
        own = cache.attend_segment(model.project(h, "q")[:, None], table, lengths)
        out = layer.merge_segments([prompt, own], B, x)
        logits = model.logits(out.view(B * x, d_m))
        logprob, entropy, top, index = el_attn.score_tokens(logits, tokens.reshape(-1).to(torch.int32).cuda(), k=2 * x)
        torch.cuda.synchronize()
        # every beam's scores against the whole history of that beam
        exact = np.stack([model.exact(H[r // x, :lens[r // x]], history[r]) for r in range(B * x)])
        ref = oracle.score_tokens_reference(exact, [t[-1] for t in history], 2 * x)
        # the step's own bars (2e-3 of the largest output in 16-bit storage, 1e-5 in fp32; here the projected keys, values and queries are
        # rounded to the storage type besides: two more roundings of a 16-bit type per score and value, half a step of 2^-8 or 2^-11 each),
        # carried into a logit: the bound of out's error times the l2 norm of an embedding, d_m^(1/2), and of out
        tol_out = {"f32": 1e-5, "f16": 2e-3 + 4 * 2.0 ** -11, "bf16": 2e-3 + 4 * 2.0 ** -8}[dtype]
        scale = tol_out * np.abs(exact).max()
        err = [np.abs(logits.cpu().numpy() - exact).max() / np.abs(exact).max(), np.abs(logprob.cpu().numpy() - ref[0]).max(),
               np.abs(top.cpu().numpy() - ref[2]).max()]
        record(f"search {dtype} step {step}: logits {err[0]:.2e} of the largest, logprob {err[1]:.2e}, top {err[2]:.2e} (bars {tol_out:.2e}, {2 * scale:.2e})")
        assert err[0] <= tol_out and err[1] <= 2 * scale and err[2] <= 2 * scale
        # the alternatives are those of the very logits that were scored
        again = oracle.score_tokens_reference(logits.cpu().numpy(), None, 2 * x)
        assert np.array_equal(index.cpu().numpy(), again[3])
        # the best of all beams of a sentence
        score = (total[:, :, None] + top.cpu().view(B, x, 2 * x)).reshape(B, -1)
        total, best = torch.topk(score, x, dim=1)
        parents = (best // (2 * x) + torch.arange(B)[:, None] * x).reshape(-1)
        tokens = torch.gather(index.cpu().view(B, -1), 1, best).long()
        pages.fork(parents.tolist())
        history = [history[int(p)] + [int(t)] for p, t in zip(parents, tokens.reshape(-1))]
    assert forks > 0, "no beam forked"
    layer.close()


def test_a_captured_step_replays_to_the_eager_result():
    """Append, attention and scores in one graph; new tokens, tables and lengths in the same buffers, eager work in between."""
    import torch
    from paper_2105_04779_amd import el_attn
    g = torch.Generator(device="cuda").manual_seed(5)
    B, x, heads, kv, d, page, cols, V = 5, 2, 8, 4, 128, 16, 200, 30011
    pool = torch.randn((2, B * cols + 3, page, kv, d), generator=g, device="cuda").to(torch.bfloat16)
    eager_pool = pool.clone()
    cache, eager = el_attn.PagedCache(pool[0], pool[1]), el_attn.PagedCache(eager_pool[0], eager_pool[1])
    table = torch.zeros((B, cols), dtype=torch.int32, device="cuda")
    lengths = torch.ones(B, dtype=torch.int32, device="cuda")
    q = torch.zeros((B, x, heads, d), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((B, 1, kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    src, dst = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))
    logits = torch.zeros((B * x, V), dtype=torch.bfloat16, device="cuda")
    tokens = torch.zeros(B * x, dtype=torch.int32, device="cuda")

    def step(c):
        c.copy_pages(src, dst)
        c.append(k, v, table, lengths)
        return (*c.attend_segment(q, table, lengths, window=2900), *el_attn.score_tokens(logits, tokens, k=11))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache)                                                  # warm-up outside the capture
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    pool.copy_(eager_pool)
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(cache)
    with torch.cuda.graph(other, pool=graph.pool()):                 # a second graph on the same memory pool
        outs2 = step(cache)
    for rep in range(4):
        order = torch.randperm(B * cols + 3, generator=g, device="cuda").to(torch.int32)
        table.copy_(order[:B * cols].view(B, cols))
        src.copy_(order[:2])
        dst.copy_(order[-2:])
        lengths.copy_(torch.tensor([1 + rep, 3200 - rep, 16 * rep + 1, 0, 777], dtype=torch.int32))
        for t in (q, k, v, logits):
            t.normal_(generator=g)
        tokens.random_(0, V, generator=g)
        torch.cuda.synchronize()
        which, got = (graph, outs) if rep % 2 == 0 else (other, outs2)
        which.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in got]
        want = step(eager)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), f"replay {rep}"
        assert torch.equal(pool, eager_pool)
