"""GPU parity of the paged cache in 8 bits (append, copies, attention) against the references.

Append and copies are exact: the definition is in fp32 operations, each rounded once.

Error bound of the attention, u = 2^-24, element by element, as for the cache in 16 bits: codes, scales and queries enter their products exactly (an fp32
query as three parts that add up to it), so a score is a sum of at most 3 d products, each addition rounded once, and scaled: off by at most
D = (3 d + 4) u max_t scale sum |q k| + 8 u max|s|.  With every score off by at most D the output is off by 2 D sum p |V|.  Sums of n positive terms add
n / 8 + 64 roundings (8 positions a lane and 32 a tile are summed at a time, then partial sums); the split of p into bf16 parts is off by 2^-16 where the result has 16
bits and 2^-23 where it has 32; the result is rounded once, by half a step of its type.  Log-sum-exp: D, the sums, 4 u |lse|.
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
NAN_CODE = {"e4m3": 127, "int8": -128}                               # what no position names holds it, with a scale of NaN


def codes_to_device(codes, fmt, heads_first=False):
    import torch
    c = codes.transpose(0, 2, 1, 3) if heads_first else codes
    t = torch.from_numpy(np.ascontiguousarray(c)).cuda()
    t = t if fmt == "int8" else t.view(torch.float8_e4m3fn)
    return t.transpose(1, 2) if heads_first else t


def codes_of(t, fmt):
    import torch
    return t.contiguous().view(torch.uint8 if fmt == "e4m3" else torch.int8).cpu().numpy()


class Case:
    """A pool, a table and queries; pages in random order; codes and scales that no position names are NaN (the largest negative number)."""

    def __init__(self, seed, fmt, dtype, B, x, heads, kv, d, page, block, lengths, heads_first=False, spare=2, query_pad=0, spread=1.0):
        import torch
        from paper_2105_04779_amd import el_attn
        g = np.random.default_rng(seed)
        self.fmt, self.dtype, self.B, self.x, self.heads, self.kv, self.d, self.page, self.block = fmt, dtype, B, x, heads, kv, d, page, block
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
        blocks = named.reshape(pages, page // block, block).any(2)
        self.pools = []
        for _ in range(2):
            if fmt == "int8":
                codes = g.integers(-127, 128, (pages, page, kv, d)).astype(np.int8)
            else:
                codes = g.integers(0, 127, (pages, page, kv, d)).astype(np.uint8) | (g.integers(0, 2, (pages, page, kv, d)) << 7).astype(np.uint8)
            # scales of all sizes; values are about 1 at most
            scale = (2.0 ** (spread * g.uniform(-3, 0, (pages, kv, page // block))) / oracle.LARGEST_CODE[fmt] * 2).astype(np.float32)
            codes[~named] = NAN_CODE[fmt]
            scale[~blocks[:, None, :].repeat(kv, 1)] = np.nan
            self.pools.append((codes, scale))
        self.q = wl.round_to_storage(g.standard_normal((B, x, heads, d), dtype=np.float32) * np.float32(2), dtype)
        self.slopes = (2.0 ** (-8.0 * (np.arange(heads) + 1) / heads)).astype(np.float32)
        (K, ks), (V, vs) = self.pools
        self.cache = el_attn.PagedCache8(codes_to_device(K, fmt, heads_first), codes_to_device(V, fmt, heads_first), torch.from_numpy(ks).cuda(), torch.from_numpy(vs).cuda())
        self.table_d, self.lengths_d = torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lengths).cuda()
        wide = np.full((B, x, heads + query_pad, d), np.nan, dtype=np.float32)
        wide[:, :, :heads] = self.q
        self.q_d = to_device(np.ascontiguousarray(wide), dtype)[:, :, :heads]

    def values(self, i):
        codes, scale = self.pools[i]
        return oracle.quantized_values(codes, self.fmt) * scale.astype(np.float64).repeat(self.block, 2).transpose(0, 2, 1)[..., None]

    def check(self, tag, out_dtype=None, segment=False, n=None, slopes=False, scale=None, **rule):
        import torch
        scale_ = self.d ** -0.5 if scale is None else scale
        ref, ref_lse, info = oracle.paged_attend_reference(self.values(0), self.values(1), self.table, self.lengths, self.q, scale=scale_, n=n,
                                                           slopes=self.slopes if slopes else None, **rule)
        kw = dict(n=n, scale=scale, slopes=torch.from_numpy(self.slopes).cuda() if slopes else None, **rule)
        if segment:
            A, lse = self.cache.attend_segment(self.q_d, self.table_d, self.lengths_d, **kw)
            got, out_dtype = A.cpu().numpy().reshape(ref.shape), "f32"
        else:
            got = self.cache.attend(self.q_d, self.table_d, self.lengths_d, out_dtype=out_dtype, **kw).float().cpu().numpy()
            out_dtype = out_dtype or self.dtype
        torch.cuda.synchronize()
        D = (3 * self.d + 4) * U * info["qk"] + 8 * U * info["s"]
        sums = (info["n"] / 8 + 64) * U
        split = {"f32": 2.0 ** -23}.get(out_dtype, 2.0 ** -16)
        bound = (2 * D + 2 * sums + split)[..., None] * info["spread"] * 1.01
        bound = bound + HALF_STEP[out_dtype] * (np.abs(ref) + bound) + SMALLEST[out_dtype] + 1e-37
        assert np.isfinite(got).all(), f"{tag}: not finite"
        worst = float((np.abs(got - ref) / bound).max())
        line = f"{tag}: {worst:.3f} of the bound, {np.abs(got - ref).max():.2e} absolute"
        if segment:
            lse = lse.cpu().numpy().reshape(ref_lse.shape)
            empty = np.isneginf(ref_lse)
            assert np.array_equal(np.isneginf(lse), empty) and not got[empty].any()
            err = np.abs(lse[~empty] - ref_lse[~empty]) / (D + sums + 4 * U * np.abs(ref_lse) + 1e-37)[~empty]
            line += f", lse {err.max() if err.size else 0:.3f} of its bound"
            assert not err.size or err.max() <= 1.0, line
        record(line)
        assert worst <= 1.0, line


FORMATS, DTYPES = ["e4m3", "int8"], ["bf16", "f16", "f32"]
LENGTHS = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 130]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,block", [(1, 1), (7, 7), (8, 8), (16, 16), (16, 8), (16, 1), (24, 24), (24, 12), (40, 8), (64, 16), (128, 128)])
def test_lengths_round_tiles_pages_and_blocks(fmt, page, block):
    c = Case(11 + page + block, fmt, "bf16", len(LENGTHS), 1, 4, 2, 64, page, block, LENGTHS)
    c.check(f"lengths {fmt} page {page} block {block}")
    c.check(f"lengths {fmt} page {page} block {block} segment", segment=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,d,x", [(1, 1, 16, 1), (3, 3, 48, 1), (6, 2, 64, 2), (8, 8, 64, 3), (34, 1, 64, 1), (7, 1, 80, 5), (16, 4, 96, 4), (8, 1, 128, 2), (33, 1, 128, 1),
                                          (9, 1, 128, 7), (2, 2, 256, 1), (10, 2, 240, 4), (40, 2, 256, 5)])
def test_head_layouts(fmt, dtype, heads, kv, d, x):
    c = Case(21 + heads, fmt, dtype, 3, x, heads, kv, d, 16, 16, [1, 75, 211])
    c.check(f"heads {heads}/{kv} d {d} x {x} {dtype} {fmt}")
    c.check(f"heads {heads}/{kv} d {d} x {x} {dtype} {fmt} segment", segment=True)
    c = Case(22 + heads, fmt, dtype, 2, x, heads, kv, d, 10, 5, [43, 75])      # pages and blocks that no 8 positions fit
    c.check(f"heads {heads}/{kv} d {d} x {x} {dtype} {fmt} odd pages", out_dtype="f32")


RULES = [dict(softcap=5.0), dict(window=1), dict(window=20), dict(window=1000), dict(slopes=True), dict(softcap=0.5, window=45, slopes=True),
         dict(scale=0.0), dict(scale=-0.3, slopes=True), dict(scale=2.0)]


@pytest.mark.parametrize("fmt,dtype,page,block", [("e4m3", "bf16", 24, 24), ("int8", "f32", 24, 24), ("int8", "f16", 12, 4)])
@pytest.mark.parametrize("rule", RULES, ids=lambda r: "-".join(f"{k}{v}" for k, v in r.items()))
def test_score_rules(fmt, dtype, page, block, rule):
    c = Case(31, fmt, dtype, 5, 2, 8, 4, 64, page, block, [0, 1, 30, 200, 333])
    c.check(f"rule {rule} {dtype} {fmt}", segment=True, **rule)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_long_caches_are_split_and_joined(fmt, dtype):
    c = Case(41, fmt, dtype, 2, 1, 4, 2, 128, 64, 64, [9000, 41])
    c.check(f"long {dtype} {fmt}", out_dtype="f32")
    c.check(f"long {dtype} {fmt} window", segment=True, window=5000, slopes=True)
    c = Case(42, fmt, dtype, 1, 1, 2, 2, 64, 16, 8, [20011])
    c.check(f"one long {dtype} {fmt}", segment=True)
    c = Case(43, fmt, dtype, 1, 2, 4, 2, 256, 20, 4, [5003])
    c.check(f"one long, odd pages {dtype} {fmt}")


@pytest.mark.parametrize("fmt", FORMATS)
def test_many_sequences_of_very_different_lengths(fmt):
    g = np.random.default_rng(7)
    for B, top in ((70, 700), (300, 90), (1100, 40)):
        lengths = (g.random(B) ** 4 * top).astype(int)
        c = Case(50 + B, fmt, "bf16", B, 1, 2, 1, 64, 16, 16, lengths)
        c.check(f"{B} sequences {fmt}", segment=True)
        c.check(f"{B} sequences {fmt}, no n", n=int(lengths.max()) + 1 if lengths.max() < c.table.shape[1] * 16 else None, out_dtype="f32")


@pytest.mark.parametrize("fmt", FORMATS)
def test_scales_of_very_different_size(fmt):
    c = Case(61, fmt, "f32", 4, 2, 4, 2, 64, 16, 8, [1, 40, 130, 500], spread=12.0)      # 2^-36 to 1
    c.check(f"spread scales {fmt}", segment=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_absent_pages_layouts_and_strides(fmt):
    import torch
    c = Case(71, fmt, "bf16", 3, 2, 8, 4, 64, 16, 8, [100, 64, 33], heads_first=True, query_pad=5)
    c.check(f"heads first {fmt}")
    for b, j, page in ((0, 2, -1), (0, 6, 10 ** 6), (1, 0, -5), (2, 2, c.cache.K.shape[0])):
        c.table[b, j] = page
    c.table_d.copy_(torch.from_numpy(c.table))
    c.check(f"absent pages {fmt}", segment=True)
    c.check(f"absent pages {fmt} window", segment=True, window=40)
    c.table[:] = -1
    c.table_d.copy_(torch.from_numpy(c.table))
    c.check(f"nothing there {fmt}", segment=True)
    c = Case(72, fmt, "f16", 3, 1, 4, 2, 128, 32, 16, [-3, 50, 200], query_pad=2)
    c.lengths_d.copy_(torch.tensor([-3, 50, 10 ** 9], dtype=torch.int32))
    c.lengths = np.array([-3, 50, c.table.shape[1] * 32])
    for pool in c.pools:                                             # (the whole table's room is there)
        held = c.table[2]
        pool[0][held] = np.where(pool[0][held] == NAN_CODE[fmt], 1, pool[0][held])
        pool[1][held] = np.nan_to_num(pool[1][held], nan=0.01)
    from paper_2105_04779_amd import el_attn
    (K, ks), (V, vs) = c.pools
    c.cache = el_attn.PagedCache8(codes_to_device(K, fmt), codes_to_device(V, fmt), torch.from_numpy(ks).cuda(), torch.from_numpy(vs).cuda())
    c.check(f"lengths outside {fmt}", segment=True)


def test_nan_and_infinite_queries_make_their_own_rows_nan():
    import torch
    for dtype in DTYPES:
        c = Case(81, "e4m3", dtype, 2, 2, 4, 2, 64, 16, 16, [40, 70])
        q = c.q_d.clone()
        q[0, 1, 2, 5], q[1, 0, 0, 0] = float("nan"), float("inf")
        out = c.cache.attend(q, c.table_d, c.lengths_d)
        want = c.cache.attend(c.q_d, c.table_d, c.lengths_d)
        torch.cuda.synchronize()
        bad = torch.zeros(out.shape[:3], dtype=torch.bool)
        bad[0, 1, 2] = bad[1, 0, 0] = True
        assert torch.isnan(out[bad.cuda()]).all() and torch.equal(out[~bad.cuda()], want[~bad.cuda()])


def test_a_given_output_another_stream_and_the_same_bits_again():
    import torch
    c = Case(82, "int8", "bf16", 40, 2, 16, 4, 128, 16, 16, np.random.default_rng(3).integers(1, 600, 40))
    first = c.cache.attend(c.q_d, c.table_d, c.lengths_d)
    out = torch.empty_like(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = c.cache.attend(c.q_d, c.table_d, c.lengths_d, out=out)
    torch.cuda.synchronize()
    assert again is out and torch.equal(out, first)
    with pytest.raises(ValueError):
        c.cache.attend(c.q_d, c.table_d, c.lengths_d, out=out[:, :1])
    with pytest.raises(ValueError):
        c.cache.attend(c.q_d.to(torch.float64), c.table_d, c.lengths_d)
    with pytest.raises(ValueError):
        c.cache.attend(c.q_d, c.table_d.long(), c.lengths_d)


# ---- append and copies ---------------------------------------------------------------------------------------------------
def _append_case(seed, fmt, dtype, B, T, kv, d, page, block, lengths, counts, tweak=None, pad=0):
    import torch
    from paper_2105_04779_amd import el_attn
    g = np.random.default_rng(seed)
    lengths = np.asarray(lengths)
    cols = max(1, int(-(-max(lengths.max(), 1) // page)))
    pages = B * cols + 2
    table = g.permutation(pages)[:B * cols].reshape(B, cols).astype(np.int32)
    pools = []
    for _ in range(2):
        codes = g.integers(-127, 128, (pages, page, kv, d)).astype(np.int8) if fmt == "int8" else \
            (g.integers(0, 127, (pages, page, kv, d)) | g.integers(0, 2, (pages, page, kv, d)) << 7).astype(np.uint8)
        pools.append((codes, (2.0 ** g.uniform(-12, -4, (pages, kv, page // block))).astype(np.float32)))
    new = [wl.round_to_storage(g.standard_normal((B, T, kv, d), dtype=np.float32) * (2.0 ** g.uniform(-3, 3, (B, T, 1, 1))).astype(np.float32), dtype) for _ in range(2)]
    if tweak:
        tweak(table, new)
        new = [wl.round_to_storage(x, dtype) for x in new]
    dev = [codes_to_device(c, fmt) for c, _ in pools] + [torch.from_numpy(s).cuda() for _, s in pools]
    cache = el_attn.PagedCache8(*dev)
    wide = [np.full((B, T, kv * d + pad), np.nan, np.float32) for _ in new]
    for w, x in zip(wide, new):
        w[..., :kv * d] = x.reshape(B, T, kv * d)
    k, v = (to_device(w, dtype)[..., :kv * d].unflatten(-1, (kv, d)) for w in wide)
    L = torch.from_numpy(lengths.astype(np.int32)).cuda()
    C = None if counts is None else torch.from_numpy(np.asarray(counts, np.int32)).cuda()
    cache.append(k, v, torch.from_numpy(table).cuda(), L, counts=C)
    torch.cuda.synchronize()
    for name, codes_d, scale_d, (codes, scale), x in (("K", dev[0], dev[2], pools[0], new[0]), ("V", dev[1], dev[3], pools[1], new[1])):
        want, want_scale = oracle.quantized_append_reference(codes, scale, table, lengths, counts, x, block, fmt)
        got_scale = scale_d.cpu().numpy()
        assert np.array_equal(got_scale, want_scale, equal_nan=True), f"{name}: scales differ at {np.argwhere(got_scale != want_scale)[:3].tolist()}"
        got = codes_of(codes_d, fmt)
        if fmt == "e4m3":                                            # (two codes are NaN)
            got, want = np.where(got == 255, 127, got), np.where(want == 255, 127, want)
        differ = np.argwhere(got != want)
        assert differ.size == 0, f"{name}: codes differ at {differ[:3].tolist()}"


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_append_is_the_definition(fmt, dtype):
    _append_case(1, fmt, dtype, 6, 1, 3, 32, 16, 16, [1, 2, 16, 17, 40, 33], None)                        # a token each: first, later, block's last
    _append_case(2, fmt, dtype, 5, 1, 2, 64, 8, 4, [1, 5, 8, 9, 31], None, pad=16)
    _append_case(3, fmt, dtype, 3, 50, 2, 48, 16, 8, [50, 90, 61], [50, 7, 33])                           # prompts, ragged, over blocks begun before
    _append_case(4, fmt, dtype, 2, 9, 1, 16, 5, 5, [9, 14], None, pad=16)
    _append_case(5, fmt, dtype, 2, 40, 1, 256, 64, 64, [40, 75], [40, 31])                                # blocks that a wavefront does not hold at once
    _append_case(6, fmt, dtype, 3, 6, 2, 16, 6, 1, [6, 11, 12], [6, 6, 2])                                # a scale for every position


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_drops_what_has_no_place_and_survives_values_without_size(fmt):
    def tweak(table, new):
        table[0, 1], table[1, 0], table[2, 0] = -1, 10 ** 6, -7
        new[0][3, 0, 0, :] = 0                                       # a block of zeros: the smallest scale
        new[0][3, 1, 0, 3], new[1][3, 2, 1, 4], new[1][4, 0, 0, 0] = np.nan, np.inf, -np.inf
        new[1][4, 1] = np.nan                                        # nothing finite
        new[0][4] *= np.float32(1e-38)
    _append_case(7, fmt, "f32", 6, 4, 2, 32, 8, 2, [12, 4, 3, 4, 4, 20], [4, 9, 4, 4, -2, 2], tweak)
    _append_case(8, fmt, "bf16", 6, 4, 2, 32, 8, 8, [12, 4, 3, 4, 2, 20], [4, 9, 4, 4, 4, 0], tweak)      # (4 of 2: two lie before the first position)


@pytest.mark.parametrize("fmt", FORMATS)
def test_tokens_one_at_a_time_have_the_scale_of_all_at_once(fmt):
    import torch
    from paper_2105_04779_amd import el_attn
    g = torch.Generator(device="cuda").manual_seed(4)
    k = torch.randn((2, 21, 2, 64), generator=g, device="cuda", dtype=torch.float16)
    v = torch.randn((2, 21, 2, 64), generator=g, device="cuda", dtype=torch.float16)
    table = torch.tensor([[3, 0], [1, 2]], dtype=torch.int32, device="cuda")
    caches = []
    for _ in range(2):
        pool = torch.zeros((2, 4, 16, 2, 64), dtype=torch.int8, device="cuda")
        pool = pool if fmt == "int8" else pool.view(torch.float8_e4m3fn)
        caches.append(el_attn.PagedCache8(pool[0], pool[1], torch.zeros((4, 2, 2), device="cuda"), torch.zeros((4, 2, 2), device="cuda")))
    caches[0].append(k, v, table, torch.full((2,), 21, dtype=torch.int32, device="cuda"))
    for t in range(21):
        caches[1].append(k[:, t:t + 1], v[:, t:t + 1], table, torch.full((2,), t + 1, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    a, b = caches
    assert torch.equal(a.K_scale, b.K_scale) and torch.equal(a.V_scale, b.V_scale)
    # rounded again at most 8 times: each is off by half a step of the scale of that time, all of them below the last
    step = {"int8": 0.5, "e4m3": 448 * 2.0 ** -4}[fmt]
    assert (a.K.float() - b.K.float()).abs().max() <= (1 + 8) * step


@pytest.mark.parametrize("fmt", FORMATS)
def test_copies_take_codes_and_scales(fmt):
    import torch
    from paper_2105_04779_amd import el_attn
    for seed, page, block, kv, d, heads_first in ((1, 16, 4, 3, 64, False), (2, 7, 7, 2, 16, False), (3, 64, 64, 4, 128, True), (4, 10, 1, 1, 256, False)):
        g = np.random.default_rng(seed)
        pages = 40
        codes = g.integers(-127, 128, (pages, page, kv, d)).astype(np.int8 if fmt == "int8" else np.uint8)
        scale = g.random((pages, kv, page // block), dtype=np.float32)
        order = g.permutation(pages)
        src, dst = order[:14].astype(np.int32), order[20:34].astype(np.int32)
        src[3], src[4], dst[5], src[6] = src[2], -1, pages, dst[6]
        counts = g.integers(-1, page + 2, 14).astype(np.int32)
        counts[:3] = 0, 1, page
        for c in (counts, None):
            K, V = codes_to_device(codes, fmt, heads_first), codes_to_device(codes[::-1].copy(), fmt, heads_first)
            ks, vs = torch.from_numpy(scale).cuda(), torch.from_numpy(scale[::-1].copy()).cuda()
            cache = el_attn.PagedCache8(K, V, ks, vs)
            cache.copy_pages(torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda(), None if c is None else torch.from_numpy(c).cuda())
            torch.cuda.synchronize()
            for t, s, c0, s0 in ((K, ks, codes, scale), (V, vs, codes[::-1], scale[::-1])):
                want, want_scale = oracle.quantized_copy_reference(c0, s0, src, dst, c, block)
                assert np.array_equal(codes_of(t, fmt), want) and np.array_equal(s.cpu().numpy(), want_scale)


def test_no_work_is_no_error_and_derivatives_are_refused():
    import torch
    c = Case(91, "e4m3", "bf16", 2, 1, 2, 2, 64, 16, 16, [5, 20])
    empty = torch.empty((0, 1), dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert c.cache.attend(c.q_d[:0], empty, none).shape == (0, 1, 2, 64)
    c.cache.append(c.q_d[:0], c.q_d[:0], empty, none)
    c.cache.copy_pages(none, none)
    q = c.q_d.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        c.cache.attend(q, c.table_d, c.lengths_d)
    with pytest.raises(ValueError):
        c.cache.append(c.q_d, c.q_d.half(), c.table_d, c.lengths_d)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_append_to_large_blocks_with_and_without_infinities(fmt, dtype):
    def tweak(table, new):
        new[0][0, 190, 0, 100], new[0][1, 3, 1, 7], new[1][0, 150, 1, 111] = np.inf, np.nan, -np.inf    # in what a wavefront holds, and behind it
        new[1][1, 40:60] = np.nan
    _append_case(11, fmt, dtype, 2, 200, 2, 112, 128, 128, [200, 331], [200, 177], tweak, pad=16)
    _append_case(12, fmt, dtype, 2, 200, 2, 112, 256, 64, [203, 331], [199, 200], pad=48)
    _append_case(13, fmt, dtype, 1, 70, 3, 80, 64, 32, [75], None, tweak=lambda table, new: new[0].__setitem__((0, 33, 2, 79), np.nan))


@pytest.mark.parametrize("fmt", FORMATS)
def test_pools_whose_offsets_pass_32_bits(fmt):
    """Pages 1.7 GB apart: the same bits as in a compact pool."""
    import torch
    from paper_2105_04779_amd import el_attn
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 25 GB of device memory")
    g = torch.Generator(device="cuda").manual_seed(9)
    B, kv, d, page, block, pages, apart = 2, 2, 128, 16, 16, 6, 1_700_000_000 // 16 * 16
    element = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    shape, strides = (pages, page, kv, d), (apart, kv * d, d, 1)
    table = torch.tensor([[5, 0, 3], [2, 4, 1]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([45, 34], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((B, 45, kv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((B, 1, 8, d), generator=g, device="cuda").to(torch.bfloat16)
    results = []
    for far in (False, True):
        K, V = (torch.as_strided(torch.empty((pages - 1) * apart + page * kv * d, dtype=torch.uint8, device="cuda").view(element), shape, strides) if far
                else torch.empty(shape, dtype=torch.uint8, device="cuda").view(element) for _ in range(2))
        scales = [torch.zeros((pages, kv, page // block), device="cuda") for _ in range(2)]
        cache = el_attn.PagedCache8(K, V, *scales)
        cache.append(k, v, table, lengths, counts=lengths)
        before = cache.attend(q, table, lengths)
        cache.copy_pages(torch.tensor([5], dtype=torch.int32, device="cuda"), torch.tensor([2], dtype=torch.int32, device="cuda"))
        after = cache.attend(q, table, lengths)
        torch.cuda.synchronize()
        results.append((before, after, *scales))
        del cache, K, V
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert not torch.equal(results[0][0][1], results[0][1][1])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_results_in_16_bits_are_those_in_32_rounded_once(fmt, dtype):
    """Whatever the result's type, sums and probabilities are the same numbers: with probabilities in fewer bits one result in a thousand was rounded the other way."""
    import torch
    element = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    for k, (B, x, heads, kv, d, page, lengths) in enumerate([(1, 1, 16, 16, 64, 16, [613]), (40, 1, 32, 8, 128, 16, list(range(1, 1600, 40))), (2, 5, 8, 1, 128, 24, [70, 999]),
                                                             (3, 1, 4, 2, 256, 8, [1, 500, 3001]), (5, 2, 4, 4, 96, 10, [9, 100, 33, 700, 0]), (1, 1, 8, 2, 128, 64, [30001])]):
        c = Case(200 + k, fmt, dtype, B, x, heads, kv, d, page, page, lengths)
        got = c.cache.attend(c.q_d, c.table_d, c.lengths_d)
        want = c.cache.attend(c.q_d, c.table_d, c.lengths_d, out_dtype="f32")
        torch.cuda.synchronize()
        differ = int((got != want.to(element)).sum())
        assert got.dtype == element and differ == 0, f"case {k}: {differ} of {got.numel()}"


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page,block,kv,d", [(16, 8, 2, 64), (16, 16, 3, 32), (10, 5, 1, 48), (8, 1, 2, 16)])
def test_tokens_one_at_a_time_are_the_definition_after_every_token(fmt, dtype, page, block, kv, d):
    """Blocks whose scale grows with every token, now and then or never: codes are rounded again as the reference rounds them, token by token, to the last code."""
    import torch
    from paper_2105_04779_amd import el_attn
    g = np.random.default_rng(100 + page + block)
    B, T = 4, 2 * page + 3
    size = np.stack([2.0 ** (np.arange(T) % block * 0.7), 2.0 ** (-np.arange(T) * 0.3), 2.0 ** g.uniform(-6, 6, T), np.ones(T)])
    new = [wl.round_to_storage((g.standard_normal((B, T, kv, d)) * size[..., None, None]).astype(np.float32), dtype) for _ in range(2)]
    pages = 3 * B + 1
    table = g.permutation(pages)[:3 * B].reshape(B, 3).astype(np.int32)
    pools = [(g.integers(0, 120, (pages, page, kv, d)).astype(np.int8 if fmt == "int8" else np.uint8), g.random((pages, kv, page // block), dtype=np.float32)) for _ in range(2)]
    dev = [codes_to_device(c, fmt) for c, _ in pools] + [torch.from_numpy(s.copy()).cuda() for _, s in pools]
    cache = el_attn.PagedCache8(*dev)
    k, v = (to_device(x, dtype) for x in new)
    table_d, again = torch.from_numpy(table).cuda(), 0
    for t in range(T):
        lengths = np.array([t + 1] * B)
        cache.append(k[:, t:t + 1], v[:, t:t + 1], table_d, torch.from_numpy(lengths.astype(np.int32)).cuda())
        torch.cuda.synchronize()
        for i in range(2):
            codes, scale = oracle.quantized_append_reference(*pools[i], table, lengths, None, new[i][:, t:t + 1], block, fmt)
            again += int((codes != pools[i][0]).any((2, 3)).sum()) - B
            pools[i] = codes, scale
            assert np.array_equal(dev[2 + i].cpu().numpy(), scale), (t, i)
            assert np.array_equal(codes_of(dev[i], fmt), codes), (t, i)
    record(f"token by token {fmt} {dtype} page {page} block {block}: {again} positions rounded again")
    assert block == 1 or again > 20
