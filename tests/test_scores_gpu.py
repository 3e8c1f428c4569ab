"""GPU parity of the token scores against the fp64 reference.

Error bound, u = 2^-24: a difference to the largest logit m is rounded once and its exponential is good to 3 u (1 + |x - m|); sums of V
positive terms in fp32 add at most V / 256 + 80 roundings; log S and the results round a few times more at their own size.  So log S
is off by D = u (3 (1 + A) + V / 256 + 80 + 4 |log S|), A = sum p |x - m|, a log-probability (x - m) - log S by that and 2 u |logprob|, whatever m
is, and the entropy by D (2 + A) for the weighted sum.  Indices are exact: the logits themselves are compared.
"""
import numpy as np
import pytest

import oracle
from paper_2105_04779_amd import workloads as wl
from helpers import record, to_device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _lse_bound(x, away):
    x = x.astype(np.float64)
    m = np.array([r[np.isfinite(r)].max() if np.isfinite(r).any() else 0.0 for r in x])
    with np.errstate(all="ignore"):
        log_s = np.array([np.log(np.exp(np.where(np.isfinite(r), r - b, -np.inf)).sum()) if np.isfinite(r).any() else 0.0
                          for r, b in zip(x, m)])
    return U * (3 * (1 + away) + x.shape[1] / 256 + 80 + 4 * np.abs(log_s))


def _check(tag, x, dtype, k, tokens="mixed", pad=0, offset=0):
    import torch
    from paper_2105_04779_amd import el_attn
    rows, V = x.shape
    g = np.random.default_rng(V)
    x = wl.round_to_storage(x, dtype)
    wide = np.full((rows, V + pad), np.float32(9e4 if dtype != "f16" else 6e4), dtype=np.float32)      # what is between rows would win
    wide[:, :V] = x
    flat = np.concatenate([np.full(offset, wide[0, -1] if pad else 0, np.float32), wide.reshape(-1)])
    dev = to_device(wl.round_to_storage(flat, dtype), dtype)[offset:].view(rows, V + pad)[:, :V]
    t = None if tokens is None else g.integers(0, V, rows).astype(np.int32) if isinstance(tokens, str) else np.asarray(tokens, np.int32)
    got = el_attn.score_tokens(dev, None if t is None else torch.from_numpy(t).cuda(), k=k)
    torch.cuda.synchronize()
    logprob, entropy, top, index = (None if y is None else y.cpu().numpy() for y in got)
    r_logprob, r_entropy, r_top, r_index, away = oracle.score_tokens_reference(x, t, k)
    assert (logprob is None) == (t is None) and top.shape == index.shape == (rows, k)
    assert np.array_equal(index, r_index), f"{tag}: indices differ in rows {np.nonzero((index != r_index).any(1))[0][:5]}"
    D = _lse_bound(x, away)
    worst = 0.0

    def close(name, y, ref, bound):
        nonlocal worst
        same = (np.isnan(y) & np.isnan(ref)) | (y == ref)
        with np.errstate(invalid="ignore"):
            ratio = np.where(same, 0.0, np.abs(y - ref) / bound)
        worst = max(worst, float(np.max(ratio, initial=0.0)))
        assert (ratio <= 1.0).all(), f"{tag}: {name} {np.nanmax(ratio)} of the bound"
    if t is not None:
        close("logprob", logprob, r_logprob, D + 2 * U * np.abs(np.nan_to_num(r_logprob, neginf=0.0)))
    close("entropy", entropy, r_entropy, D * (2 + away))
    close("top", top, r_top, D[:, None] + 2 * U * np.abs(np.nan_to_num(r_top, neginf=0.0)))
    record(f"{tag}: {worst:.3f} of the bound")


def _logits(seed, rows, V, scale=2.0):
    return np.random.default_rng(seed).standard_normal((rows, V), dtype=np.float32) * np.float32(scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,V,k", [(1, 1, 1), (2, 2, 5), (3, 7, 7), (4, 63, 64), (1, 255, 3), (5, 257, 8), (3, 1000, 64), (4, 2049, 8), (2, 8191, 20),
                                      (4, 16385, 10), (3, 50265, 8), (1, 131072, 64), (2, 200003, 50), (70, 4099, 4)])
def test_sizes(dtype, rows, V, k):
    _check(f"{dtype} {rows}x{V} k {k}", _logits(V, rows, V), dtype, k)


@pytest.mark.parametrize("dtype,rows,V,k", [("bf16", 300, 33333, 8), ("f16", 600, 16001, 64), ("f32", 257, 20011, 20), ("bf16", 1100, 4097, 3), ("f32", 280, 70001, 5),
                                            ("bf16", 256, 131072, 2), ("f32", 3, 524288, 64), ("bf16", 2, 524287, 64)])
def test_many_rows_and_the_largest_vocabulary(dtype, rows, V, k):
    _check(f"{dtype} {rows}x{V} k {k}", _logits(V + rows, rows, V), dtype, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (7, 3), (64, 1), (0, 5)])
def test_rows_that_start_anywhere(dtype, pad, offset):
    _check(f"{dtype} pad {pad} offset {offset}", _logits(3, 6, 5003), dtype, 12, pad=pad, offset=offset)
    _check(f"{dtype} pad {pad} offset {offset} short", _logits(4, 6, 5), dtype, 3, pad=pad, offset=offset)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_ties_and_orders(dtype):
    V = 40000
    rows = [np.zeros(V), np.full(V, -3.5), np.linspace(0, 9, V), np.linspace(9, 0, V), np.where(np.arange(V) % 2, -0.0, 0.0),
            np.where(np.arange(V) < V - 3, -60000.0, 1.0), np.where(np.arange(V) % 997 == 5, 2.0, 1.0), np.where(np.arange(V) >= V - 900, 4.0, -4.0),
            np.repeat(np.linspace(5, 4, 10), V // 10)]
    x = np.stack(rows).astype(np.float32)
    for k in (1, 8, 64):
        _check(f"ties {dtype} k {k}", x, dtype, k)
    # rows that are cut: ties within a chunk and across chunks
    for k in (1, 64):
        _check(f"ties, cut {dtype} k {k}", np.tile(x, (1, 7)), dtype, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,offset", [(1500, 0), (33337, 3), (120001, 5), (300007, 1)])
def test_thousands_of_ties_at_the_bound(dtype, V, offset):
    """More elements tie than are ranked by counting: some larger ones before and behind, ties from a place on, a few lanes' only, at both ends of a
    row that starts anywhere, all of one sign of zero or both."""
    g = np.random.default_rng(V)
    x = np.zeros((10, V), dtype=np.float32)
    x[1] = np.minimum(g.standard_normal(V), 0)
    x[2, g.permutation(V)[:5]] = (3.0, 1.0, 2.0, 1.0, 7.0)
    x[3, :V // 3] = -1
    x[4] = -2.5
    x[4, :3], x[4, -4:] = 1.0, 1.0
    x[5, ::2] = -0.0
    x[6] = np.where(np.arange(V) % 2048 < 16, 1.0 + (np.arange(V) % 7), -np.inf)     # a few lanes hold all
    x[7] = np.where(np.arange(V) < V - 1100, -np.inf, 4.0)
    x[8, V // 2:V // 2 + 1200] = g.integers(1, 4, len(x[8, V // 2:V // 2 + 1200]))
    x[9, g.permutation(V)[:40]] = 1.0
    for k in (1, 8, 64):
        _check(f"ties at the bound {dtype} V {V} k {k}", x, dtype, k, pad=7, offset=offset)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("k", [1, 8, 20, 64])
def test_alternatives_of_rows_that_are_cut(dtype, k):
    """All in one chunk, one in each, in none but a few places, nowhere."""
    V = 300001
    g = np.random.default_rng(k)
    x = np.full((7, V), -np.inf, dtype=np.float32)
    x[0] = np.linspace(-9, 9, V)
    x[1] = x[0, ::-1]
    x[2, g.permutation(V)[:3]] = (1.0, 5.0, -2.0)
    x[3, ::5003] = g.standard_normal(len(x[3, ::5003]))
    x[5] = g.standard_normal(V) * 4
    x[5, 123456:123500] += 40
    x[6, 170000:170060] = g.standard_normal(60)
    _check(f"cut {dtype} k {k}", x, dtype, k)


@pytest.mark.parametrize("dtype,rows,V", [("bf16", 4, 50265), ("f32", 300, 30011), ("bf16", 2, 250000)])
def test_results_repeat_to_the_bit(dtype, rows, V):
    """Which lane writes an alternative is a matter of chance; what it writes is not."""
    import torch
    from paper_2105_04779_amd import el_attn
    x = to_device(wl.round_to_storage(_logits(13, rows, V), dtype), dtype)
    t = torch.arange(rows, dtype=torch.int32, device="cuda")
    once = el_attn.score_tokens(x, t, k=20)
    for _ in range(20):
        for a, b in zip(once, el_attn.score_tokens(x, t, k=20)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_banned_tokens(dtype):
    g = np.random.default_rng(8)
    x = _logits(9, 8, 30011)
    x[0, :] = -np.inf                                                # none may follow
    x[1, 1:] = -np.inf
    x[2, :-1] = -np.inf
    x[3, g.random(30011) < 0.999] = -np.inf                          # about 30
    x[4, 20000:] = -np.inf
    x[5, :20000] = -np.inf
    x[6, :] = -np.inf
    x[6, [3, 16390, 29000]] = [1.0, 1.0, 2.0]
    for k in (1, 5, 40):
        _check(f"banned {dtype} k {k}", x, dtype, k, tokens=[7, 0, 30010, 5, 25000, 25000, 3, 9])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_extreme_logits(dtype):
    big = 60000.0
    x = _logits(10, 7, 9001)
    x[0, 77] = big                                                   # certain
    x[1, :] = -big                                                   # large and equal
    x[2, 5] = np.nan
    x[3, 9] = np.inf
    x[4] *= 50
    x[5, 4000:] = -big                                               # the lowest of the type as a mask
    x[6, :] = np.nan
    _check(f"extreme {dtype}", x, dtype, 6, tokens=[77, 3, 5, 9, 1, 5000, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows", [1, 40])
def test_masks_of_the_types_lowest_value(dtype, rows):
    """A finite mask leaves a distribution, over all of a row if all is masked; so do logits of any size.  Vocabularies of one launch and of two."""
    low = {"bf16": -3.3895313892515355e38, "f16": -65504.0, "f32": -3.4028234663852886e38}[dtype]
    for V in (5003, 300007):
        x = np.tile(_logits(14, 8, V), (rows, 1))[:, :V]
        x[0::8] = low                                                # uniform
        x[1::8, 7:] = low
        x[2::8] = -low                                               # the highest
        x[3::8, 100] = -low
        if dtype != "f16":
            x[4::8] = -1e9
            x[5::8] += 1e6
            x[6::8] *= 1e30
        x[7::8, V // 2:] = low
        x = x[:max(rows, 8)]
        _check(f"lowest {dtype} V {V}", x, dtype, 12, tokens=np.arange(len(x)) % V)


def test_tokens_that_are_none():
    x = _logits(11, 5, 777)
    _check("no token", x, "f32", 3, tokens=[-1, 776, 777, -2147483648, 2147483647])
    _check("no tokens at all", x, "f32", 0, tokens=None)


def test_rows_beyond_32_bits_of_elements():
    """Three rows 2^31 elements apart, 8.6 GB of bf16, and the same rows one behind the other.  The two start at other places between
    16-byte boundaries, so their sums are taken in another order and need not have the same bits: each result is within its bound of
    the exact one, so the two are within twice that of each other.  The indices are the same."""
    import torch
    from paper_2105_04779_amd import el_attn
    V, step = 5003, 1 << 31
    flat = torch.zeros(2 * step + V, dtype=torch.bfloat16, device="cuda")
    x = wl.round_to_storage(_logits(12, 3, V), "bf16")
    rows = flat.as_strided((3, V), (step, 1))
    rows.copy_(to_device(x, "bf16"))
    t = torch.tensor([1, 2, 5002], dtype=torch.int32, device="cuda")
    far, near = el_attn.score_tokens(rows, t, k=9), el_attn.score_tokens(to_device(x, "bf16"), t, k=9)
    ref = oracle.score_tokens_reference(x, t.cpu().numpy(), 9)
    D = _lse_bound(x, ref[4])
    bounds = (D + 2 * U * np.abs(ref[0]), D * (2 + ref[4]), D[:, None] + 2 * U * np.abs(ref[2]))
    for a, b, bound in zip(far, near, bounds):
        assert (np.abs(a.cpu().numpy() - b.cpu().numpy()) <= 2 * bound).all()
    assert torch.equal(far[3], near[3]) and np.array_equal(far[3].cpu().numpy(), ref[3])


def test_refusals():
    import torch
    from paper_2105_04779_amd import el_attn
    x = torch.zeros((4, 100), device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: el_attn.score_tokens(x.double(), t), lambda: el_attn.score_tokens(x[0], t), lambda: el_attn.score_tokens(x.t(), t),
                 lambda: el_attn.score_tokens(x, t.long()), lambda: el_attn.score_tokens(x, t[:2]), lambda: el_attn.score_tokens(x, t.cpu()),
                 lambda: el_attn.score_tokens(x, t, k=65), lambda: el_attn.score_tokens(x, t, k=-1),
                 lambda: el_attn.score_tokens(x.requires_grad_(), t)):
        with pytest.raises(ValueError):
            call()
            pytest.fail("taken")
