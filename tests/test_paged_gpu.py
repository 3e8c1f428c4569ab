"""GPU parity of the paged key/value cache (attention of one new token over pages, append, copies) against the fp64 references.

Error bound of the attention, u = 2^-24 (fp32), element by element.  A score is a product of fp32 sums: off by at most
(d + 4) u max_t scale sum |q k| for the products and 8 u max|s| for scale, cap, bias and the conversion to a power of two (tanh
and the exponential instruction are good to 2 ulp; neither has a slope beyond 1).  With every score off by at most D, every
probability is off by a factor within e^(2 D), the output by 2 D sum p |V|.  Sums of n positive terms in fp32 add n / 16 + 64
roundings (16 positions are summed at a time, then partial sums), the split of p into 16-bit parts 2^-16 where the result itself has 16 bits and 2^-23
where it has 32, and the result is rounded once, by half a step of its type.  Log-sum-exp: D, the sums, 4 u |lse|.
"""
import numpy as np
import pytest

import oracle
from paper_2105_04779_amd import workloads as wl
from helpers import record, to_device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
SMALLEST = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}             # half a step among the subnormal numbers


def _host(t):
    return t.float().cpu().numpy()


class Case:
    """A pool, a table and queries; pages in random order, every place that no position names holds NaN."""

    def __init__(self, seed, dtype, B, x, heads, kv, d, page, lengths, heads_first=False, spare=2, query_pad=0):
        import torch
        from paper_2105_04779_amd import el_attn
        g = np.random.default_rng(seed)
        self.dtype, self.B, self.x, self.heads, self.kv, self.d, self.page = dtype, B, x, heads, kv, d, page
        lengths = np.asarray(lengths, dtype=np.int64)
        cols = max(1, int(-(-max(lengths.max(), 1) // page)))
        held = [-(-int(max(n, 0)) // page) for n in lengths]
        pages = sum(held) + spare
        order = g.permutation(pages)
        self.table = np.full((B, cols), -1, dtype=np.int32)
        named = np.zeros((pages, page), bool)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = order[at:at + h]
            for t in range(int(max(lengths[b], 0))):
                named[self.table[b, t // page], t % page] = True
            at += h
        self.lengths = lengths.astype(np.int32)
        draw = lambda *s: wl.round_to_storage(g.standard_normal(s, dtype=np.float32), dtype)
        self.K, self.V = draw(pages, page, kv, d), draw(pages, page, kv, d)
        self.K[~named] = np.nan
        self.V[~named] = np.nan
        self.q = draw(B, x, heads, d)
        self.slopes = (2.0 ** (-8.0 * (np.arange(heads) + 1) / heads)).astype(np.float32)
        to = lambda a: to_device(np.ascontiguousarray(a), dtype)
        if heads_first:
            Kd, Vd = to(self.K.transpose(0, 2, 1, 3)).transpose(1, 2), to(self.V.transpose(0, 2, 1, 3)).transpose(1, 2)
        else:
            Kd, Vd = to(self.K), to(self.V)
        self.cache = el_attn.PagedCache(Kd, Vd)
        self.table_d, self.lengths_d = torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lengths).cuda()
        wide = np.full((B, x, heads + query_pad, d), np.nan, dtype=np.float32)
        wide[:, :, :heads] = self.q
        self.q_d = to(wide)[:, :, :heads]

    def check(self, tag, out_dtype=None, segment=False, n=None, slopes=False, scale=None, **rule):
        import torch
        scale_ = self.d ** -0.5 if scale is None else scale
        ref, ref_lse, info = oracle.paged_attend_reference(self.K, self.V, self.table, self.lengths, self.q, scale=scale_, n=n,
                                                           slopes=self.slopes if slopes else None, **rule)
        kw = dict(n=n, scale=scale, slopes=torch.from_numpy(self.slopes).cuda() if slopes else None, **rule)
        if segment:
            A, lse = self.cache.attend_segment(self.q_d, self.table_d, self.lengths_d, **kw)
            got, out_dtype = _host(A).reshape(ref.shape), "f32"
        else:
            got = _host(self.cache.attend(self.q_d, self.table_d, self.lengths_d, out_dtype=out_dtype, **kw))
            out_dtype = out_dtype or self.dtype
        torch.cuda.synchronize()
        D = (self.d + 4) * U * info["qk"] + 8 * U * info["s"]
        sums = (info["n"] / 16 + 64) * U
        split = {"f32": 2.0 ** -23}.get(out_dtype, 2.0 ** -16)
        bound = (2 * D + 2 * sums + split)[..., None] * info["spread"] * 1.01
        bound = bound + HALF_STEP[out_dtype] * (np.abs(ref) + bound) + SMALLEST[out_dtype] + 1e-37
        assert np.isfinite(got).all(), f"{tag}: not finite"
        worst = float((np.abs(got - ref) / bound).max())
        line = f"{tag}: {worst:.3f} of the bound, {np.abs(got - ref).max():.2e} absolute"
        if segment:
            lse = _host(lse).reshape(ref_lse.shape)
            empty = np.isneginf(ref_lse)
            assert np.array_equal(np.isneginf(lse), empty) and not got[empty].any()
            err = np.abs(lse[~empty] - ref_lse[~empty]) / (D + sums + 4 * U * np.abs(ref_lse) + 1e-37)[~empty]
            line += f", lse {err.max() if err.size else 0:.3f} of its bound"
            assert not err.size or err.max() <= 1.0, line
        record(line)
        assert worst <= 1.0, line


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 130]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_lengths_round_tiles_and_pages(dtype, page):
    c = Case(11 + page, dtype, len(LENGTHS), 1, 4, 2, 64, page, LENGTHS)
    c.check(f"lengths {dtype} page {page}")
    c.check(f"lengths {dtype} page {page} segment", segment=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("heads,kv,d,x", [(1, 1, 8, 1), (3, 3, 16, 1), (6, 2, 40, 2), (8, 8, 64, 3), (7, 1, 80, 5), (16, 4, 96, 4), (8, 1, 128, 2),
                                          (33, 1, 128, 1), (9, 1, 128, 7), (2, 2, 256, 1), (10, 2, 248, 4), (40, 2, 256, 5)])
def test_head_layouts(dtype, heads, kv, d, x):
    c = Case(21 + heads, dtype, 3, x, heads, kv, d, 16, [1, 75, 211])
    c.check(f"heads {heads}/{kv} d {d} x {x} {dtype}")
    c.check(f"heads {heads}/{kv} d {d} x {x} {dtype} segment", segment=True)


RULES = [dict(softcap=5.0), dict(window=1), dict(window=20), dict(window=1000), dict(slopes=True), dict(softcap=0.5, window=45, slopes=True),
         dict(scale=0.0), dict(scale=-0.3, slopes=True), dict(scale=2.0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rule", RULES, ids=lambda r: "-".join(f"{k}{v}" for k, v in r.items()))
def test_score_rules(dtype, rule):
    c = Case(31, dtype, 5, 2, 8, 4, 64, 24, [0, 1, 30, 200, 333])
    c.check(f"rule {rule} {dtype}", segment=True, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_long_caches_are_split_and_joined(dtype):
    c = Case(41, dtype, 2, 1, 4, 2, 128, 64, [9000, 41])
    c.check(f"long {dtype}", out_dtype="f32")
    c.check(f"long {dtype} window", segment=True, window=5000, slopes=True)
    c = Case(42, dtype, 1, 1, 2, 2, 64, 16, [20011])
    c.check(f"one long {dtype}", segment=True)


def test_many_sequences_of_very_different_lengths():
    g = np.random.default_rng(7)
    lengths = np.where(g.random(300) < 0.02, g.integers(1500, 4000, 300), g.integers(0, 40, 300))
    c = Case(43, "bf16", 300, 1, 2, 2, 64, 16, lengths)
    c.check("300 ragged", segment=True)
    c = Case(44, "f16", 1500, 1, 2, 1, 64, 16, g.integers(0, 50, 1500))
    c.check("1500 ragged")


@pytest.mark.parametrize("dtype,d,heads,kv,x", [("bf16", 8, 2, 1, 1), ("f16", 40, 4, 4, 1), ("bf16", 80, 8, 2, 5), ("f32", 96, 3, 1, 1), ("f16", 248, 2, 2, 1),
                                                ("f32", 256, 2, 1, 9), ("f32", 20, 2, 1, 17), ("bf16", 128, 20, 1, 2)])
def test_cut_sequences_of_every_width(dtype, d, heads, kv, x):
    """Few long sequences, whose many pieces are joined by four wavefronts a row, and many, by one, with spans that go on from one
    sequence to the next, empty ones among them."""
    c = Case(52, dtype, 2, x, heads, kv, d, 16, [5000, 2100])
    c.check(f"cut, few {dtype} d {d}", segment=True, window=4000)
    g = np.random.default_rng(d)
    lengths = np.where(g.random(70) < 0.2, 0, g.integers(1, 2200, 70))
    lengths[-1] = 2150
    c = Case(53, dtype, 70, x, heads, kv, d, 16, lengths)
    c.check(f"cut, many {dtype} d {d}")
    lengths[[7, 69]] = (4500, 4200)
    c = Case(59, dtype, 70, x, heads, kv, d, 16, lengths)
    c.check(f"cut, many, longer {dtype} d {d}", segment=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_short_sequences_taken_whole(dtype):
    g = np.random.default_rng(8)
    c = Case(54, dtype, 640, 1, 4, 4, 64, 16, g.integers(0, 200, 640))
    c.check(f"640 whole {dtype}", segment=True)


@pytest.mark.parametrize("dtype,kv", [("bf16", 700), ("f32", 1500)])
def test_key_heads_that_do_not_divide_the_device_evenly(dtype, kv):
    c = Case(55, dtype, 2, 1, kv, kv, 16, 16, [700, 333])
    c.check(f"{kv} key heads {dtype}", segment=True)


@pytest.mark.parametrize("B,kv,d", [(1100, 2, 32), (4200, 1, 8), (16390, 1, 8)])
def test_thousands_of_sequences_with_a_few_long_ones(B, kv, d):
    """Cut by sums over blocks of lengths, of more than 64 each among them, and past the number that is cut."""
    g = np.random.default_rng(B)
    lengths = g.integers(0, 4, B)
    lengths[[0, 63, 64, 700, B - 2]] = (4100, 5, 900, 4250, 1300)
    lengths[B - 40:B - 2] = 0
    lengths[B - 1] = 0
    c = Case(58, "f16", B, 1, kv, kv, d, 64, lengths)
    c.check(f"{B} sequences", segment=True)
    c.check(f"{B} sequences, window", window=1500)


@pytest.mark.parametrize("dtype,B,kv,d,x", [("bf16", 643, 8, 64, 1), ("f16", 8, 9, 64, 3), ("f16", 300, 9, 24, 1), ("bf16", 13, 5, 40, 7), ("f32", 259, 8, 20, 1), ("f32", 300, 8, 32, 1)])
def test_heads_that_share_lines_of_memory(dtype, B, kv, d, x):
    """Many heads and sequences in both layouts, numbers of them that divide nothing, a few rows each or enough for several blocks."""
    g = np.random.default_rng(B)
    for i, heads_first in enumerate((False, True)):
        c = Case(56 + i, dtype, B, x, 3 * kv, kv, d, 16, g.integers(0, 180, B), heads_first=heads_first)
        c.check(f"{B} x {kv} heads of {d} {dtype}", segment=True)


def test_lengths_outside_the_call_are_taken_as_the_nearer_end():
    c = Case(45, "bf16", 4, 1, 4, 4, 64, 16, [300, 7, 0, 160])
    c.lengths = np.array([400, -3, -2147483648, 2147483647], dtype=np.int32)
    c.table[:, :] = c.table[0]                                       # every sequence on the first one's pages
    import torch
    c.table_d, c.lengths_d = torch.from_numpy(c.table).cuda(), torch.from_numpy(c.lengths).cuda()
    c.check("outside, n 300", n=300, segment=True)
    c.check("outside, n 33", n=33, segment=True)
    # no lengths: n for all
    got = c.cache.attend(c.q_d, c.table_d, None, n=33)
    c.lengths = np.array([33] * 4, dtype=np.int32)
    c.lengths_d = torch.from_numpy(c.lengths).cuda()
    assert torch.equal(got, c.cache.attend(c.q_d, c.table_d, c.lengths_d, n=33))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_absent_pages_and_pages_out_of_the_pool(dtype):
    import torch
    c = Case(46, dtype, 4, 1, 4, 2, 64, 8, [100, 100, 40, 64])
    c.table[0, [0, 5, 12]] = [-1, 10 ** 6, -2147483648]
    c.table[1, :] = -1                                               # nothing at all
    c.table[2, 1:] = c.K.shape[0]                                    # one past the pool
    c.table[3, :7] = 2147483647
    c.table_d = torch.from_numpy(c.table).cuda()
    c.check(f"absent {dtype}", segment=True)
    c.check(f"absent {dtype} window", segment=True, window=30)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_pages_and_other_layouts(dtype):
    import torch
    c = Case(47, dtype, 3, 2, 6, 3, 96, 16, [90, 77, 100], heads_first=True, query_pad=5)
    c.table[1, :4] = c.table[0, :4]                                  # a shared prefix
    c.table_d = torch.from_numpy(c.table).cuda()
    c.check(f"heads first, shared {dtype}", segment=True)
    # a slice of a wider pool (every second position and the upper half of the heads), a slice of a wider table
    from paper_2105_04779_amd import el_attn
    K = torch.full((c.K.shape[0], 32, 6, 96), float("nan"), device="cuda", dtype=c.q_d.dtype)
    V = K.clone()
    K[:, ::2, 3:], V[:, ::2, 3:] = to_device(c.K, dtype), to_device(c.V, dtype)
    c.cache = el_attn.PagedCache(K[:, ::2, 3:], V[:, ::2, 3:])
    wide = torch.full((3, 20), -1, dtype=torch.int32, device="cuda")
    wide[:, 4:4 + c.table.shape[1]] = c.table_d
    c.table_d = wide[:, 4:4 + c.table.shape[1]]
    c.check(f"slices {dtype}", segment=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_infinite_and_extreme_scores(dtype):
    """Keys of -inf (a score of -inf is a position that takes no part), values of inf where a probability is 0, scores that reach the
    top of the type, a NaN that has to come out."""
    import torch
    c = Case(48, dtype, 4, 1, 2, 2, 64, 16, [50, 50, 50, 50])
    q = np.abs(c.q) + 0.5
    c.q = wl.round_to_storage(q, dtype)
    c.q_d = to_device(c.q, dtype)
    K, V = c.cache.K, c.cache.V
    K[c.table[0, 1], :, :, :] = -float("inf")                        # 16 positions at -inf
    c.K[c.table[0, 1]] = -np.inf
    for j in range(4):                                               # all positions at -inf
        K[c.table[1, j], :, :, :] = -float("inf")
        c.K[c.table[1, j]] = -np.inf
    V[c.table[0, 1], :, :, :] = 7.0
    c.V[c.table[0, 1]] = 7.0
    big = wl.round_to_storage(c.K[c.table[2, 0], 3] * 0 + np.float32(100.0), dtype)
    K[c.table[2, 0], 3] = 100.0                                      # one score hundreds above the rest
    c.K[c.table[2, 0], 3] = big
    K[c.table[3, 2], 5, 1] = float("nan")
    ref, ref_lse, _ = oracle.paged_attend_reference(c.K[:, :, :, :], c.V, c.table, c.lengths[:3], c.q[:3], scale=0.125)
    A, lse = c.cache.attend_segment(c.q_d, c.table_d, c.lengths_d)
    A, lse = _host(A).reshape(4, 2, 64), _host(lse)
    assert not A[1].any() and np.isneginf(lse[1]).all()
    for b in (0, 2):
        assert np.abs(A[b] - ref[b, 0]).max() < 1e-4 * np.abs(ref[b]).max() and np.abs(lse[b] - ref_lse[b, 0]).max() < 1e-4 * np.abs(ref_lse[b]).max()
    assert np.isnan(A[3, 1]).all() and np.isnan(lse[3, 1]) and np.isfinite(A[3, 0]).all() and np.isfinite(lse[3, 0])


def test_caches_beyond_32_bits_of_elements():
    """Pages whose elements lie more than 2^32 elements apart, bf16: 10 GB of pool."""
    import torch
    from paper_2105_04779_amd import el_attn
    pages, page, kv, d = 9, 16, 2, 64
    pool = torch.zeros(2 * (1 << 32) + (1 << 28), dtype=torch.bfloat16, device="cuda")
    stride = 1 << 29                                                 # elements between pages: page 8 starts at 2^32
    K = pool.as_strided((pages, page, kv, d), (stride, kv * d, d, 1))
    V = pool.as_strided((pages, page, kv, d), (stride, kv * d, d, 1), 1 << 28)
    c = Case(49, "bf16", 1, 1, 4, 2, 64, 16, [9 * 16 - 3], spare=0)
    K.copy_(to_device(c.K, "bf16"))
    V.copy_(to_device(c.V, "bf16"))
    c.cache = el_attn.PagedCache(K, V)
    c.check("strides of 2^29 elements", segment=True)
    # the same places through append and copy
    new = torch.randn((1, 1, kv, d), device="cuda").to(torch.bfloat16)
    last = c.table_d.clone()
    last[0, 0] = 8
    c.cache.append(new, new * 2, last, torch.tensor([1], dtype=torch.int32, device="cuda"))
    assert torch.equal(K[8, 0], new[0, 0]) and torch.equal(V[8, 0], new[0, 0] * 2)
    c.cache.copy_pages(torch.tensor([8], dtype=torch.int32, device="cuda"), torch.tensor([7], dtype=torch.int32, device="cuda"))
    assert torch.equal(K[7].nan_to_num(5.0), K[8].nan_to_num(5.0)) and torch.equal(V[7].nan_to_num(5.0), V[8].nan_to_num(5.0))


def test_results_repeat_and_streams_keep_apart():
    """The same call twice gives the same bits; two calls at once on two streams, each with its own scratch memory, as well."""
    import torch
    c = Case(50, "bf16", 6, 2, 8, 2, 128, 16, [4000, 17, 900, 0, 2500, 3])
    d = Case(51, "bf16", 6, 2, 8, 2, 128, 16, [3, 1700, 90, 4000, 250, 0])
    once = [k.cache.attend_segment(k.q_d, k.table_d, k.lengths_d) for k in (c, d)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        twice = []
        for k, s in zip((c, d), streams):
            with torch.cuda.stream(s):
                twice.append(k.cache.attend_segment(k.q_d, k.table_d, k.lengths_d))
        torch.cuda.synchronize()
        for (A, S), (A2, S2) in zip(once, twice):
            assert torch.equal(A, A2) and torch.equal(S, S2)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,T,kv,d,page", [(1, 1, 1, 8, 1), (5, 1, 8, 64, 16), (3, 40, 2, 80, 7), (2, 513, 4, 128, 32), (70, 3, 1, 256, 16),
                                             (3, 259, 1, 8, 16), (2, 100, 3, 24, 5), (4, 31, 1, 64, 16), (2, 9, 17, 256, 4)])
def test_append(dtype, B, T, kv, d, page):
    import torch
    g = np.random.default_rng(60 + T)
    lengths = g.integers(0, 2 * T + 3, B)
    lengths[0] = T + 2
    c = Case(61, dtype, B, 1, kv, kv, d, page, lengths)
    new = [wl.round_to_storage(g.standard_normal((B, T, kv, d), dtype=np.float32), dtype) for _ in range(2)]
    # from a fused projection: a token's keys and values among other columns
    fused = torch.zeros((B, T, 3 * kv * d + 16), device="cuda", dtype=c.q_d.dtype)
    fused[..., :kv * d] = to_device(new[0], dtype).reshape(B, T, -1)
    fused[..., 2 * kv * d:3 * kv * d] = to_device(new[1], dtype).reshape(B, T, -1)
    k, v = fused[..., :kv * d].unflatten(2, (kv, d)), fused[..., 2 * kv * d:3 * kv * d].unflatten(2, (kv, d))
    for counts in (None, g.integers(-1, T + 2, B)):
        K, V = c.cache.K.clone(), c.cache.V.clone()
        want = oracle.paged_append_reference(_host(K), _host(V), c.table, lengths, counts, *new)
        c.cache.append(k, v, c.table_d, c.lengths_d, counts=None if counts is None else torch.from_numpy(counts.astype(np.int32)).cuda())
        torch.cuda.synchronize()
        for got, w in zip((c.cache.K, c.cache.V), want):
            np.testing.assert_array_equal(_host(got), w)             # (NaN where nothing was written, as before)


def test_append_drops_what_has_no_place():
    import torch
    c = Case(62, "bf16", 5, 1, 2, 2, 64, 4, [10, 10, 10, 10, 10])
    c.table[1, 1], c.table[2, 2], c.table[3, 0] = -1, 10 ** 9, -2147483648
    lengths = np.array([13, 10, 10, 2, -2147483648], dtype=np.int32)
    g = np.random.default_rng(63)
    new = [wl.round_to_storage(g.standard_normal((5, 9, 2, 64), dtype=np.float32), "bf16") for _ in range(2)]
    want = oracle.paged_append_reference(c.K, c.V, c.table, lengths, None, *new)
    c.cache.append(to_device(new[0], "bf16"), to_device(new[1], "bf16"), torch.from_numpy(c.table).cuda(), torch.from_numpy(lengths).cuda())
    for got, w in zip((c.cache.K, c.cache.V), want):
        np.testing.assert_array_equal(_host(got), w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv,d,page,heads_first", [(1, 8, 1, False), (16, 64, 16, False), (3, 80, 7, True), (2, 256, 64, True), (8, 128, 33, False)])
def test_copy_pages(dtype, kv, d, page, heads_first):
    import torch
    c = Case(70, dtype, 1, 1, kv, kv, d, page, [page * 8], heads_first=heads_first, spare=8)
    pages = c.K.shape[0]
    g = np.random.default_rng(71)
    order = g.permutation(pages)
    src, dst = order[[0, 1, 2, 2, 3, 4]].astype(np.int32), order[[8, 9, 10, 11, 12, 4]].astype(np.int32)   # one source twice, one page to itself
    src[4] = pages
    for counts in (None, np.array([page, 1, page // 2, page + 5, page, 1], dtype=np.int32), np.array([0, -4, 1, page, 1, 1], dtype=np.int32)):
        want = oracle.paged_copy_reference(_host(c.cache.K), _host(c.cache.V), src, dst, counts)
        c.cache.copy_pages(torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda(), counts=None if counts is None else torch.from_numpy(counts).cuda())
        for got, w in zip((c.cache.K, c.cache.V), want):
            np.testing.assert_array_equal(_host(got), w)


def test_binding_refusals():
    import torch
    from paper_2105_04779_amd import el_attn
    c = Case(80, "bf16", 2, 2, 4, 2, 64, 16, [20, 33])
    t, n, q = c.table_d, c.lengths_d, c.q_d
    bad = [lambda: c.cache.attend(q.float(), t, n), lambda: c.cache.attend(q[..., :32], t, n), lambda: c.cache.attend(q[:, :, :3], t, n),
           lambda: c.cache.attend(q, t.long(), n), lambda: c.cache.attend(q, t[:1], n), lambda: c.cache.attend(q, t, n.long()),
           lambda: c.cache.attend(q, t, n[:1]), lambda: c.cache.attend(q, t.cpu(), n), lambda: c.cache.attend(q, t.t().contiguous().t(), n),
           lambda: c.cache.attend(q.transpose(0, 1), t, n), lambda: c.cache.attend(q, t, n, slopes=torch.ones(3, device="cuda")),
           lambda: c.cache.attend(q, t, n, slopes=torch.ones(4, device="cuda", dtype=torch.float64)),
           lambda: c.cache.attend(q, t, n, out=torch.empty_like(q, dtype=torch.float32)),
           lambda: c.cache.attend(q.clone().requires_grad_(), t, n),
           lambda: c.cache.append(q[:, :, :2], q[:, :, :2], t, n.long()), lambda: c.cache.append(q, q, t, n),
           lambda: c.cache.append(q[:, :, :2], q[:, :, :2].contiguous(), t, n), lambda: c.cache.append(q[:, :, :2].float(), q[:, :, :2].float(), t, n),
           lambda: c.cache.copy_pages(n, n[:1]), lambda: c.cache.copy_pages(n.long(), n.long()),
           lambda: el_attn.PagedCache(c.cache.K, c.cache.V.float()), lambda: el_attn.PagedCache(c.cache.K[0], c.cache.V[0]),
           lambda: el_attn.PagedCache(c.cache.K, c.cache.V.transpose(1, 2).contiguous().transpose(1, 2))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    for kw in (dict(n=10 ** 6), dict(n=0), dict(window=-1), dict(softcap=-1.0), dict(scale=float("nan")), dict(out_dtype="f16")):
        with pytest.raises(el_attn.ElAttnError):
            c.cache.attend(q, t, n, **kw)
