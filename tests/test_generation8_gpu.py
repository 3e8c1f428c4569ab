"""Generation on the paged cache in 8 bits as a program runs it: the step's table, copies for sequences that fork, new tokens, attention joined with a shared
prompt's segment, the next tokens drawn.

A toy decoder of one attention layer on token embeddings.  The pools are read back through the table of every step: each position of each sequence has to hold its own
token, and the attention's results are checked against the definition on what the pools hold."""
import numpy as np
import pytest

import oracle
from paper_2105_04779_amd import workloads as wl
from helpers import device_weights, record, to_device
from test_quantized_gpu import U, codes_of

pytestmark = pytest.mark.gpu


def _pools(fmt, pages, page, kv, d, block):
    import torch
    from paper_2105_04779_amd import el_attn
    codes = torch.full((2, pages, page, kv, d), 127, dtype=torch.uint8, device="cuda")           # (NaN in e4m3)
    codes = codes.view(torch.int8) if fmt == "int8" else codes.view(torch.float8_e4m3fn)
    scales = torch.full((2, pages, kv, page // block), float("nan"), device="cuda")
    return el_attn.PagedCache8(codes[0], codes[1], scales[0], scales[1])


@pytest.mark.parametrize("fmt,dtype,heads,d_m,page,block", [("e4m3", "bf16", 8, 512, 8, 8), ("int8", "f16", 16, 1024, 4, 2), ("int8", "f32", 4, 64, 16, 8)])
def test_sampled_continuations_of_a_shared_prompt(fmt, dtype, heads, d_m, page, block):
    import torch
    from paper_2105_04779_amd import el_attn
    B, x, n, V, steps, pages = 3, 4, 60, 1013, 21, 40
    d = d_m // heads
    w = wl.custom("generation", dtype=dtype, B=1, beam=1, heads=heads, d_m=d_m, d_k=d, n=8, index=95)
    W = wl.weights(w)
    Wd = device_weights(W, dtype)
    g = np.random.default_rng(1)
    E = to_device(wl.round_to_storage(g.standard_normal((V, d_m), dtype=np.float32), dtype), dtype)
    H = to_device(wl.round_to_storage(g.standard_normal((B, n, d_m), dtype=np.float32), dtype), dtype)
    L = torch.tensor([60, 33, 7], dtype=torch.int32, device="cuda")
    layer = el_attn.ElAttention(Wd, heads=heads, d_k=d, dtype=dtype, max_batch=B * x, max_beam=x, max_n=n)
    cache = _pools(fmt, pages, page, heads, d, block)
    project = lambda h, name: (h.float() @ Wd["W" + name].float() + Wd["b" + name].float()).to(h.dtype).unflatten(-1, (heads, d))[:, None]
    rows = B * x
    table = torch.full((rows, -(-steps // page)), -1, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(rows, dtype=torch.int32, device="cuda")
    tokens = torch.tensor([7 + 3 * b for b in range(B) for _ in range(x)], dtype=torch.int32, device="cuda")
    parents, history, forks = torch.arange(rows, dtype=torch.int32, device="cuda"), [[int(t)] for t in tokens], 0
    kv_of = {}
    for step in range(steps):
        plan = el_attn.plan_pages(table, lengths, pages=pages, page_size=page, parents=parents)
        cache.copy_pages(*plan.copies)
        h = E[tokens.long()]
        k, v, q = (project(h, name) for name in "kvq")
        cache.append(k, v, plan.table, plan.lengths, plan.granted)
        own = cache.attend_segment(q, plan.table, plan.lengths)
        out = layer.merge_segments([layer.decode_segment(H, L, h.view(B, x, d_m)), own], B, x)
        logits = out.view(rows, d_m).float() @ E.float().t() / 8.0
        drawn, logprob = el_attn.sample_tokens(logits, torch.from_numpy(g.random(rows, dtype=np.float32)).cuda(), temperature=0.9, top_k=30, top_p=0.9)
        torch.cuda.synchronize()
        assert plan.granted.cpu().tolist() == [1] * rows and plan.lengths.cpu().tolist() == [step + 1] * rows
        forks += int((plan.copies[0] >= 0).sum())
        for r in range(rows):
            kv_of[history[r][-1]] = (k[r, 0].float().cpu().numpy(), v[r, 0].float().cpu().numpy())
        t, slots = plan.table.cpu().numpy(), plan.slots.cpu().numpy()
        values = []
        for name, codes, scale in (("K", cache.K, cache.K_scale), ("V", cache.V, cache.V_scale)):
            s = scale.cpu().numpy().astype(np.float64)
            c = oracle.quantized_values(codes_of(codes, fmt), fmt)
            values.append(c * s.repeat(block, 2).transpose(0, 2, 1)[..., None])
            for r in range(rows):
                for i, token in enumerate(history[r]):
                    at, o = t[r, i // page], i % page
                    want = kv_of[token][name == "V"]
                    # rounded when it came, and once more whenever its block's scale grew: at most `block` times, each by half a step of a scale no larger
                    # than the last (e4m3: 2^-4 of the value, or half the smallest step, 2^-10)
                    last = s[at, :, o // block][:, None]
                    bar = (1 + block) * (last * 0.5 if fmt == "int8" else np.maximum(np.abs(want) * 2.0 ** -4 * 1.07 ** block, last * 2.0 ** -10)) + 1e-6
                    assert (np.abs(values[-1][at, o] - want) <= bar).all(), (name, step, r, i)
                assert slots[r, 0] == t[r, step // page] * page + step % page
        ref, ref_lse, info = oracle.paged_attend_reference(values[0], values[1], t, [step + 1] * rows, q.float().cpu().numpy(), scale=d ** -0.5)
        D = (3 * d + 4) * U * info["qk"] + 8 * U * info["s"]
        sums = (info["n"] / 8 + 64) * U
        bound = (2 * D + 2 * sums + 2.0 ** -23)[..., None] * info["spread"] * 1.01 + 2.0 ** -24 * np.abs(ref) + 1e-37
        err = np.abs(own[0].cpu().numpy().reshape(ref.shape) - ref) / bound
        assert err.max() <= 1.0, f"step {step}: {err.max()} of the bound"
        assert (np.abs(own[1].cpu().numpy().reshape(ref_lse.shape) - ref_lse) <= D + sums + 4 * U * np.abs(ref_lse)).all()
        # sequences of a sentence go on from one another
        parents = torch.tensor([r // x * x + int(g.integers(0, x)) if g.random() < 0.4 else r for r in range(rows)], dtype=torch.int32, device="cuda")
        drawn = drawn.cpu()
        history = [history[int(p)] + [int(drawn[r])] for r, p in enumerate(parents.cpu())]
        tokens = drawn.cuda()
        table, lengths = plan.table, plan.lengths
    record(f"generation {fmt} {dtype}: {forks} copies, free {int(plan.free)}")
    assert forks > 0
    layer.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_captured_step_replays_to_the_eager_result(fmt):
    """Plan, copies, append, attention and sampling in one graph; new lengths, parents and tokens in the same buffers, eager work in between."""
    import torch
    from paper_2105_04779_amd import el_attn
    g = torch.Generator(device="cuda").manual_seed(5)
    B, x, heads, kv, d, page, cols, V, pages = 6, 2, 8, 4, 128, 16, 200, 30011, 700
    cache, eager = (_pools(fmt, pages, page, kv, d, 8) for _ in range(2))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    table, lengths, parents, counts = i32(B, cols), i32(B), i32(B), i32(B)
    q = torch.zeros((B, x, heads, d), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((B, 3, kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    logits, u = torch.zeros((B * x, V), dtype=torch.bfloat16, device="cuda"), torch.zeros(B * x, device="cuda")

    def step(c):
        plan = el_attn.plan_pages(table, lengths, counts, pages=pages, page_size=page, tokens=3, parents=parents)
        c.copy_pages(*plan.copies)
        c.append(k, v, plan.table, plan.lengths, plan.granted)
        return (*plan, *c.attend_segment(q, plan.table, plan.lengths, window=2900), *el_attn.sample_tokens(logits, u, top_p=0.9, temperature=0.8),
                *el_attn.sample_tokens(logits, u))

    def fill(rep):
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        n = [3, 1000, 16 * rep, 0, 77 + rep, 1600]
        held = [-(-t // page) for t in n]
        assert sum(held) <= pages
        t = torch.full((B, cols), -1, dtype=torch.int32)
        at = 0
        for b, m in enumerate(held):
            t[b, :m] = order[at:at + m].cpu()
            at += m
        table.copy_(t)
        lengths.copy_(torch.tensor(n, dtype=torch.int32))
        parents.copy_(torch.tensor([0, 1, 4, 4, 0, -1], dtype=torch.int32))
        counts.random_(0, 4, generator=g)
        for y in (q, k, v, logits):
            y.normal_(generator=g)
        u.uniform_(generator=g)
        for c in (cache, eager):                                     # the same pool on both sides, of numbers
            torch.manual_seed(rep)
            for codes, scale in ((c.K, c.K_scale), (c.V, c.V_scale)):
                codes.view(torch.uint8).copy_(torch.randint(0, 120, codes.shape, dtype=torch.uint8, device="cuda"))
                scale.copy_(torch.rand(scale.shape, device="cuda") * 0.01 + 0.001)
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache)                                                  # warm-up outside the capture
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(cache)
    with torch.cuda.graph(other, pool=graph.pool()):                 # a second graph on the same memory pool
        outs2 = step(cache)
    for rep in range(5):
        fill(rep)
        torch.cuda.synchronize()
        which, got = (graph, outs) if rep % 2 == 0 else (other, outs2)
        which.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in got]
        want = step(eager)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), f"replay {rep}"
        for a, b in ((cache.K, eager.K), (cache.V, eager.V)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(cache.K_scale, eager.K_scale) and torch.equal(cache.V_scale, eager.V_scale)
