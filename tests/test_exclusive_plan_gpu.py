"""GPU parity of the page plan of a cache in 8 bits, and what sequences that share pages hold while others write."""
import numpy as np
import pytest

import oracle
from helpers import record
from test_page_plan_gpu import _random
from test_quantized_gpu import codes_of, codes_to_device

pytestmark = pytest.mark.gpu


def _plan(table, lengths, counts, parents, reserved, pages, page_size, T):
    import torch
    from paper_2105_04779_amd import el_attn
    to = lambda a, t=np.int32: None if a is None else torch.from_numpy(np.ascontiguousarray(np.asarray(a, t))).cuda()
    return el_attn.plan_pages(to(table), to(lengths), to(counts), pages=pages, page_size=page_size, tokens=T, parents=to(parents), reserved=to(reserved, np.uint8), exclusive=True)


def _check(tag, table, lengths, counts, parents, reserved, pages, page_size, T):
    plan = _plan(table, lengths, counts, parents, reserved, pages, page_size, T)
    want = oracle.plan_pages_reference(table, lengths, counts, parents, reserved, pages, page_size, T, exclusive=True)
    for name in ("table", "lengths", "granted", "copies", "free", "slots"):
        got = getattr(plan, name).cpu().numpy()
        ref = np.reshape(want[name], got.shape)
        assert np.array_equal(got, ref), f"{tag}: {name} differs at {np.argwhere(got != ref)[:4].tolist()}"
    return want


@pytest.mark.parametrize("page_size", [1, 5, 16])
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("seed", range(4))
def test_random_plans(page_size, T, seed):
    B_old, B, columns = [(1, 1, 1), (5, 9, 12), (33, 20, 30), (300, 700, 9)][seed]       # (the last in four launches)
    copies = 0
    for k, (room, fork, absent, share, reserve) in enumerate([(1000, False, 0, 0.5, 0), (40, True, 0, 0.5, 0), (3, True, 0.2, 0.5, 0.3), (0, True, 0, 0, 0)]):
        args = _random(500 + 100 * seed + 10 * T + k + page_size, B_old, B if fork else B_old, columns, page_size, T, room, fork, absent, share, reserve)
        copies += int((_check(f"page {page_size} T {T} seed {seed} kind {k}", *args[:5], args[5], page_size, T)["copies"][0] >= 0).sum())
    record(f"exclusive plans, page {page_size} T {T} seed {seed}: {copies} copies")


def test_a_reader_keeps_its_page_and_the_last_to_write_is_refused_where_pages_are_out():
    table = np.array([[1, 2, -1], [3, 2, -1], [4, 2, -1]])
    w = _check("a reader with as many", table, [15, 15, 15], [0, 1, 0], None, None, 10, 8, 1)
    assert w["copies"].T.tolist() == [[-1, -1, 0], [2, 0, 7], [-1, -1, 0]]
    w = _check("no page for a copy", table, [15, 15, 15], [0, 1, 0], None, None, 5, 8, 1)
    assert w["granted"].tolist() == [0, 1, 0]
    w = _check("none at all", table, [15, 15, 15], [0, 1, 0], None, [1, 0, 0, 0, 0], 5, 8, 1)
    assert w["granted"].tolist() == [0, 0, 0] and w["table"][1].tolist() == [3, 2, -1]


@pytest.mark.parametrize("fmt,page,block,pages", [("int8", 8, 8, 15), ("e4m3", 8, 8, 15), ("int8", 16, 4, 11), ("e4m3", 4, 2, 25), ("int8", 5, 5, 21)])
def test_what_others_write_changes_nothing_that_a_sequence_holds(fmt, page, block, pages):
    """Sequences fork, some write a few tokens of very different size, some none, and the pool runs out now and then.  After each step every code and scale of the pools is the
    references', and a sequence that was granted nothing has the values that its parent had, bit for bit; of one that writes, the blocks that were full do."""
    import torch
    from paper_2105_04779_amd import el_attn
    g = np.random.default_rng(page + block)
    rows, kv, d, columns, T = 8, 2, 32, 64 // page + 1, 3
    pools = [(np.zeros((pages, page, kv, d), np.int8 if fmt == "int8" else np.uint8), np.ones((pages, kv, page // block), np.float32)) for _ in range(2)]
    dev = [codes_to_device(c, fmt) for c, _ in pools] + [torch.from_numpy(s).cuda() for _, s in pools]
    cache = el_attn.PagedCache8(*dev)
    table, lengths = np.full((rows, columns), -1), np.zeros(rows, int)
    silent = refused = grown = 0

    def values(pool, table, b, n):
        at, o = table[b, np.arange(n) // page], np.arange(n) % page
        return oracle.quantized_values(pool[0][at, o], fmt) * pool[1][at, :, o // block].astype(np.float64)[..., None]
    for step in range(40):
        parents = np.where(g.random(rows) < 0.35, g.integers(0, rows, rows), np.arange(rows))
        parents[g.random(rows) < 0.04] = -1
        counts = np.where(g.random(rows) < 0.3, 0, g.integers(1, T + 1, rows))
        new = [(g.standard_normal((rows, T, kv, d)) * 2.0 ** g.uniform(-3, 8, (rows, T, 1, 1))).astype(np.float32) for _ in range(2)]
        plan = _plan(table, lengths, counts, parents, None, pages, page, T)
        cache.copy_pages(*plan.copies)
        k, v = (torch.from_numpy(x).cuda() for x in new)
        cache.append(k, v, plan.table, plan.lengths, plan.granted)
        torch.cuda.synchronize()
        want = oracle.plan_pages_reference(table, lengths, counts, parents, None, pages, page, T, exclusive=True)
        assert np.array_equal(plan.table.cpu().numpy(), want["table"]) and np.array_equal(plan.granted.cpu().numpy(), want["granted"])
        before = pools
        pools = []
        for i, (codes, scale) in enumerate(before):
            codes, scale = oracle.quantized_copy_reference(codes, scale, *want["copies"], block)
            pools.append(oracle.quantized_append_reference(codes, scale, want["table"], want["lengths"], want["granted"], new[i], block, fmt))
            assert np.array_equal(codes_of(dev[i], fmt), pools[i][0]) and np.array_equal(dev[2 + i].cpu().numpy(), pools[i][1]), f"step {step}: pool {i}"
        for b, p in enumerate(parents):
            had = int(lengths[p]) if p >= 0 else 0
            same = had if want["granted"][b] == 0 else had // block * block
            for i in range(2):
                assert np.array_equal(values(pools[i], want["table"], b, same), values(before[i], table, p, same) if p >= 0 else np.zeros((0, kv, d))), f"step {step}: sequence {b}"
                grown += int(want["granted"][b] > 0 and had > same and not np.array_equal(values(pools[i], want["table"], b, had), values(before[i], table, p, had)))
            silent += int(counts[b] == 0 and had > 0)
            refused += int(counts[b] > 0 and want["granted"][b] == 0)
        table, lengths = want["table"], want["lengths"]
    record(f"exclusive plan {fmt} page {page} block {block}: {silent} silent, {refused} refused, {grown} blocks rounded again")
    assert silent > 20 and refused > 0 and grown > 20


@pytest.mark.parametrize("small", [True, False])
def test_a_captured_exclusive_plan_replays_to_the_eager_result(small):
    import torch
    from paper_2105_04779_amd import el_attn
    B, columns = (20, 12) if small else (300, 40)
    args = [_random(40 + i, B, B, columns, 16, 5, 0, True, 0.0, 0.5) for i in range(4)]
    pages = max(a[5] for a in args) + 30
    to = lambda a: torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()
    state = [to(a) for a in args[0][:4]]
    call = lambda: el_attn.plan_pages(*state[:3], pages=pages, page_size=16, tokens=5, parents=state[3], exclusive=True)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for a in args:
        for s, x in zip(state, a[:4]):
            s.copy_(to(x))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        ref = oracle.plan_pages_reference(a[0], a[1], a[2], a[3], None, pages, 16, 5, exclusive=True)
        assert np.array_equal(got[0].cpu().numpy(), ref["table"]) and np.array_equal(got[3].cpu().numpy(), ref["slots"])
