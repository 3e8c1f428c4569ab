"""GPU parity of the sampling against the fp64 reference.

Tokens are exact.  Weights are whole multiples of 2^-43 of the largest, each off by half of that and by the exponential's 2^-40 of its own size, so a sum of V of them
is off by less than 2^-38 of itself for the vocabularies here: where the reference's decisions lie further than that from going the other way (`margin`, which is
checked), the token must be the same.  The log-probability is computed in 64 bits and rounded once: 2^-24 of itself, and 2^-38.
"""
import numpy as np
import pytest

import oracle
from paper_2105_04779_amd import workloads as wl
from helpers import record, to_device

pytestmark = pytest.mark.gpu

MARGIN = 2.0 ** -38


def _check(tag, x, dtype, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, pad=0, offset=0, tight=()):
    """`tight`: rows whose decisions are exact ones (equal weights), however close."""
    import torch
    from paper_2105_04779_amd import el_attn
    rows, V = x.shape
    x = wl.round_to_storage(x, dtype)
    wide = np.full((rows, V + pad), np.float32(9e4 if dtype != "f16" else 6e4), dtype=np.float32)      # what is between rows would win
    wide[:, :V] = x
    flat = np.concatenate([np.full(offset, 5, np.float32), wide.reshape(-1)])
    dev = to_device(wl.round_to_storage(flat, dtype), dtype)[offset:].view(rows, V + pad)[:, :V]
    f = np.float32
    full = {"temperature": (temperature, f), "top_k": (top_k, np.int32), "top_p": (top_p, f), "min_p": (min_p, f)}
    given = {k: torch.from_numpy(np.asarray(v, t)).cuda() if np.ndim(v) else v for k, (v, t) in full.items()}
    per_row = {k: np.broadcast_to(np.asarray(v, t), (rows,)) for k, (v, t) in full.items()}
    uniform = np.asarray(uniform, f)
    tokens, logprob = el_attn.sample_tokens(dev, torch.from_numpy(uniform).cuda(), **given)
    torch.cuda.synchronize()
    tokens, logprob = tokens.cpu().numpy(), logprob.cpu().numpy()
    want, want_logprob, margin = oracle.sample_tokens_reference(x, uniform, **per_row)
    margin[list(tight)] = np.inf
    assert margin.min() > MARGIN, f"{tag}: the reference itself is within {margin.min():.1e} of another answer"
    assert np.array_equal(tokens, want), f"{tag}: rows {np.nonzero(tokens != want)[0][:5]}: {tokens[tokens != want][:5]} for {want[tokens != want][:5]}"
    same = (np.isnan(logprob) & np.isnan(want_logprob)) | (logprob == want_logprob)
    with np.errstate(invalid="ignore"):
        err = np.where(same, 0.0, np.abs(logprob - want_logprob) / (2.0 ** -24 * np.abs(want_logprob) + MARGIN))
    record(f"{tag}: logprob {err.max():.3f} of the bound, margin {margin.min():.1e}")
    assert (err <= 1.0).all(), f"{tag}: logprob {np.nanmax(err)} of the bound"
    return tokens


def _rows(seed, rows, V, banned=0.0):
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, V), dtype=np.float32) * np.float32(2)
    hot = g.integers(0, V, (rows, 12))
    for r in range(rows):
        x[r, hot[r]] += g.random(12, dtype=np.float32) * 10
    x[g.random((rows, V)) < banned] = -np.inf
    return x, g.random(rows, dtype=np.float32)


FILTERS = [dict(), dict(temperature=0.3), dict(temperature=1.9), dict(top_k=1), dict(top_k=7), dict(top_k=300), dict(top_p=0.5), dict(top_p=0.99), dict(min_p=0.1), dict(min_p=1.0),
           dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.02), dict(temperature=0.0), dict(top_p=1e-6), dict(top_p=0.0), dict(min_p=2.0), dict(top_k=10 ** 9, top_p=2.0, min_p=-1.0)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rule", FILTERS, ids=lambda r: "-".join(f"{k}{v}" for k, v in r.items()) or "none")
def test_filters(dtype, rule):
    for V, rows, pad, offset in ((5, 6, 3, 1), (1000, 9, 0, 0), (50265, 4, 7, 3)):
        x, u = _rows(V + rows, rows, V)
        _check(f"{rule} V {V} {dtype}", x, dtype, u, pad=pad, offset=offset, **rule)


@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 1023, 1024, 1025, 4097, 16383, 65537, 131073, 200003])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_vocabularies(V, dtype):
    x, u = _rows(V, 3, V, 0.05 if V > 3 else 0.0)
    for rule in (dict(), dict(top_p=0.9), dict(top_k=min(V, 40), temperature=0.7)):
        _check(f"V {V} {dtype} {rule}", x, dtype, u, offset=V % 3, pad=V % 5, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_settings_of_each_row(dtype):
    g = np.random.default_rng(5)
    rows, V = 64, 9001
    x, u = _rows(6, rows, V, 0.1)
    _check(f"mixed {dtype}", x, dtype, u, temperature=g.choice([0.0, 0.5, 1.0, 1.5], rows), top_k=g.choice([0, -3, 1, 20, 5000], rows),
           top_p=g.choice([0.3, 0.9, 1.0, 1.5], rows), min_p=g.choice([0.0, -1.0, 0.05, 0.5], rows))
    nan = np.full(rows, np.nan)
    _check(f"settings of NaN {dtype}", x, dtype, u, temperature=nan)
    _check(f"filters of NaN {dtype}", x, dtype, u, top_p=nan, min_p=nan)
    _check(f"an infinite temperature {dtype}", np.where(x > 0, x, -np.inf), dtype, u, temperature=np.full(rows, 1e30), tight=range(rows))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_min_p_before_and_behind_the_bound_of_top_p(dtype):
    p, m = (a.reshape(-1) for a in np.meshgrid([0.2, 0.6, 0.9, 0.99, 0.9999], [1e-7, 1e-5, 1e-3, 0.03, 0.3, 0.7, 0.99]))
    x, u = _rows(17, p.size, 20011, 0.02)
    for temperature, k in ((1.0, 0), (2.5, 0), (1.3, 900)):
        _check(f"top-p and min-p, T {temperature} k {k} {dtype}", x, dtype, u, temperature=temperature, top_k=k, top_p=p, min_p=m, pad=1)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [1, 7, 515, 4099, 30011])
def test_more_rows_than_compute_units(V, dtype):
    g = np.random.default_rng(V)
    rows = 263
    x, u = _rows(V + 1, rows, V, 0.05 if V > 7 else 0.0)
    x[5, :] = -np.inf
    x[6, V // 2] = np.nan
    x[7, :] = 1.5                                                    # one order
    x[8, :] = np.where(np.arange(V) % 2, 1.5, 1.0)
    for n, rule in enumerate((dict(), dict(top_k=40, top_p=0.9), dict(top_p=0.95), dict(top_k=300, temperature=1.7), dict(temperature=0.0),
                              dict(temperature=g.choice([0.0, 0.7, 1.0, 2.0], rows), top_k=g.choice([0, 1, 60, 200, 900], rows),
                                   top_p=g.choice([0.2, 0.8, 0.97, 1.0], rows), min_p=g.choice([0.0, 1e-4, 0.04, 0.6], rows)))):
        _check(f"{rows} rows V {V} {dtype} rule {n}", x, dtype, u, pad=n % 3, offset=n % 2, tight=(7, 8), **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_equal_logits_go_by_index(dtype):
    V = 3001
    flat = np.full((6, V), 2.5, np.float32)
    u = [0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24, 0.1]
    # weights are equal, so the token is the whole part of u times how many stay
    tokens = _check(f"flat {dtype}", flat, dtype, u, tight=range(6))
    assert tokens.tolist() == [int(np.float64(np.float32(v)) * V) for v in u]
    tokens = _check(f"flat top-k {dtype}", flat, dtype, u, top_k=10, tight=range(6))
    assert tokens.tolist() == [0, 2, 5, 7, 9, 1]
    _check(f"flat top-p {dtype}", flat, dtype, u, top_p=0.25, tight=range(6))
    _check(f"flat min-p {dtype}", flat, dtype, u, min_p=1.0, tight=range(6))
    # ties at the bound of top-k, spread over the vocabulary, some below the larger ones
    g = np.random.default_rng(9)
    x = g.choice([0.0, 1.0, 2.0, 3.0], (8, V), p=[0.5, 0.3, 0.15, 0.05]).astype(np.float32)
    for k in (1, 100, 200, 1000):
        _check(f"ties k {k} {dtype}", x, dtype, g.random(8), top_k=k, tight=range(8))
    _check(f"ties top-p {dtype}", x, dtype, g.random(8), top_p=0.37)
    zeros = np.zeros((4, V), np.float32)
    zeros[:, ::2] = -0.0
    assert _check(f"zeros of both signs {dtype}", zeros, dtype, [0.0, 0.5, 0.9, 0.99], top_k=4, tight=range(4)).tolist() == [0, 2, 3, 3]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_without_numbers(dtype):
    V = 777
    x, u = _rows(11, 8, V)
    x[0] = -np.inf
    x[1, 5] = np.nan
    x[2, 6] = np.inf
    x[3] = np.nan
    x[4] = -np.inf
    x[4, 700] = -3.0
    x[5] = -60000.0
    x[6] = np.where(np.arange(V) % 7 == 3, 60000.0, -60000.0)
    big = {"f32": 3.0e38, "bf16": 3.0e38, "f16": 65504.0}[dtype]
    x[7] = np.where(np.arange(V) % 7 == 3, big, -big)
    for rule in (dict(), dict(top_k=9), dict(top_p=0.5), dict(min_p=0.1), dict(temperature=0.0)):
        _check(f"odd rows {dtype} {rule}", x, dtype, u, tight=range(8), **rule)


def test_random_numbers_outside_their_range():
    x, _ = _rows(12, 5, 300)
    x[:, :2] = -np.inf
    x[:, -3:] = -np.inf
    u = np.array([-0.5, 1.0, 7.0, np.nan, 0.0], np.float32)
    tokens = _check("outside", x, "f32", u, tight=range(5))
    assert tokens.tolist() == [2, 296, 296, 296, 2]


def test_frequencies():
    """Evenly spread random numbers draw every token as often as its probability says, to one draw."""
    x, _ = _rows(13, 1, 40)
    n = 20000
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    import torch
    from paper_2105_04779_amd import el_attn
    tokens, _ = el_attn.sample_tokens(torch.from_numpy(np.repeat(x, n, 0)).cuda(), torch.from_numpy(u).cuda(), temperature=1.3)
    p = torch.softmax(torch.from_numpy(x[0]).double() / float(np.float32(1.3)), 0).numpy()
    # (u in fp32 is off by 2^-25, far below the 1 / n between two)
    assert np.abs(np.bincount(tokens.cpu().numpy(), minlength=40) - n * p).max() <= 1.0 + 1e-3


def test_refusals_and_no_rows():
    import torch
    from paper_2105_04779_amd import el_attn
    x, u = torch.zeros((4, 9), device="cuda"), torch.zeros(4, device="cuda")
    tokens, logprob = el_attn.sample_tokens(x[:0], u[:0])
    assert tokens.shape == logprob.shape == (0,)
    for bad in (dict(temperature=torch.ones(4, device="cuda", dtype=torch.float64)), dict(top_k=torch.ones(4, device="cuda")), dict(top_p=torch.ones(3, device="cuda")),
                dict(min_p=torch.ones(4)), dict(temperature=-1.0), dict(temperature=float("nan")), dict(top_k=1 << 40)):
        with pytest.raises((ValueError, el_attn.ElAttnError)):
            el_attn.sample_tokens(x, u, **bad)
    with pytest.raises(ValueError):
        el_attn.sample_tokens(x, u.double())
    with pytest.raises(ValueError):
        el_attn.sample_tokens(x, torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError, match="gradient"):
        el_attn.sample_tokens(x.clone().requires_grad_(), u)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("copies", [1, 40])                          # (40: more rows than compute units)
def test_log_probabilities_of_unlikely_tokens(dtype, copies):
    """A random number of 0 draws the first token that has a weight, however small.  Its log-probability is off by the rounding to fp32, 2^-24 of itself, and by the total's: its
    weights are off by 2^-44 and the exponential's 2^-44.6 of themselves, all of them at most 1, and the total is at least 1."""
    import torch
    from paper_2105_04779_amd import el_attn
    g = np.random.default_rng(23)
    V = 300
    gaps = np.array([3.0, 11.0, 17.5, 20.75, 23.0, 25.5, 27.25, 29.0, 30.0])
    for temperature in (1.0, 0.5, 1.75):
        for rule, banned in ((dict(), 0.0), (dict(top_k=50), 0.9), (dict(top_k=200), 0.5), (dict(min_p=5e-14), 0.0), (dict(top_k=250, min_p=5e-14), 0.3)):
            x = g.uniform(-9.0, -1.0, (len(gaps), V)) * temperature
            x[g.random(x.shape) < banned] = -np.inf
            x[:, 0], x[:, 5] = -gaps * temperature, 0.0
            x = np.repeat(wl.round_to_storage(x.astype(np.float32), dtype), copies, 0)
            assert (np.isfinite(x).sum(1) < rule.get("top_k", V + 1)).all()                # top-k leaves all
            z = x.astype(np.float64) / temperature
            want = z[:, 0] - np.log(np.exp(z).sum(1))
            tokens, logprob = el_attn.sample_tokens(to_device(x, dtype), torch.zeros(len(x), device="cuda"), temperature=temperature, **rule)
            torch.cuda.synchronize()
            assert (tokens == 0).all(), (temperature, rule)
            err = np.abs(logprob.cpu().numpy() - want) / (2.0 ** -24 * np.abs(want) + V * (2.0 ** -44 + 2.0 ** -44.6) + 2.0 ** -48)
            record(f"unlikely tokens {dtype} T {temperature} {rule}: {err.max():.3f} of the bound")
            assert err.max() <= 1.0, (temperature, rule, err.reshape(-1, copies)[:, 0])


@pytest.mark.parametrize("rows", [(1 << 22) + 5, (1 << 23) - 1, 1 << 23])
def test_as_many_rows_as_there_may_be(rows):
    """2^23 rows, workgroups of 512 lanes: more than one launch, each with its rows' settings."""
    import torch
    from paper_2105_04779_amd import el_attn
    g = torch.Generator(device="cuda").manual_seed(rows)
    V = 3
    x = torch.randint(-512, 513, (rows, V), generator=g, device="cuda").to(torch.float16) / 256      # (some ties)
    way = torch.randint(0, 6, (rows,), generator=g, device="cuda")                        # which setting leaves the largest alone, if one does
    off = torch.zeros(rows, device="cuda")
    f = lambda i, value, other: torch.where(way == i, off + value, off + other)
    tokens, logprob = el_attn.sample_tokens(x, off, temperature=f(1, 0.0, 1.0), top_k=f(2, 1, 0).to(torch.int32), top_p=f(3, 0.0, 1.0), min_p=f(4, 2.0, 0.0))
    torch.cuda.synchronize()
    z = x.double()
    first = (z == z.amax(1, keepdim=True)).to(torch.uint8).argmax(1)                      # ties: the lowest index
    alone = (way >= 1) & (way <= 4)
    assert torch.equal(tokens.long(), torch.where(alone, first, 0))                        # a random number of 0 draws the first token
    want = torch.where(alone, 0.0, z[:, 0] - torch.logsumexp(z, 1))
    assert ((logprob.double() - want).abs() <= 2.0 ** -24 * want.abs() + V * 2.0 ** -43).all()


def test_no_row_follows_from_another_launch():
    """The first and the last row of 2^22 + 5, drawn alone."""
    import torch
    from paper_2105_04779_amd import el_attn
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, V = (1 << 22) + 5, 9
    x, u = torch.randn((rows, V), generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    p = torch.rand(rows, generator=g, device="cuda")
    tokens, logprob = el_attn.sample_tokens(x, u, top_p=p)
    for at in (0, 1, (1 << 22) - 2, (1 << 22) - 1, 1 << 22, rows - 2):
        few = slice(at, at + 2)
        t, l = el_attn.sample_tokens(x[few], u[few], top_p=p[few])
        torch.cuda.synchronize()
        assert torch.equal(tokens[few], t) and torch.equal(logprob[few], l), at


def _crowded(kind, rows, V):
    """Rows most of whose logits fall into one of the 512 ranges that a bound is looked for in, more than a workgroup collects."""
    g = np.random.default_rng(31)
    normal = lambda *shape: g.standard_normal(shape)
    if kind == "near":                                               # many values, few of them equal
        x = 1.0 + 1e-3 * normal(rows, V)
    elif kind == "ties":                                             # some dozens of neighbouring fp32 numbers
        x = 1.0 + 2e-6 * normal(rows, V)
    elif kind == "two":                                              # two of such clusters: a part of a range is a range of too many again
        x = np.where(g.random((rows, V)) < 0.5, 1.0, 1.02) + 1e-6 * normal(rows, V)
    elif kind == "few":                                              # one number among its neighbours, not too many in all
        x = -9.0 + normal(rows, V)
        for r in range(rows):
            at = g.permutation(V)
            x[r, at[:2500]] = 1.0
            x[r, at[2500:2540]] = 1.0 + 2.0 ** -23 * (1 + np.arange(40) // 2)
            x[r, at[2540:2580]] = 1.0 - 2.0 ** -24 * (1 + np.arange(40) // 2)
            x[r, at[2580:2600]] = 1.0 + g.uniform(-8e-3, 8e-3, 20)
    else:                                                            # a high temperature
        x = 2.0 * normal(rows, V)
    return x.astype(np.float32), g.random(rows, dtype=np.float32), 1000.0 if kind == "hot" else 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V", [(3, 60000), (2, 200003), (259, 20011)])      # (the last: workgroups of 512 lanes)
@pytest.mark.parametrize("kind", ["near", "ties", "two", "few", "hot"])
def test_ranges_of_too_many_are_cut_again(kind, rows, V, dtype):
    x, u, temperature = _crowded(kind, rows, V)
    for rule in (dict(top_p=0.9), dict(top_p=0.03), dict(top_k=1501), dict(top_k=V // 2, top_p=0.7), dict(top_p=0.9, min_p=0.9985)):
        _check(f"crowded {kind} {rows} of {V} {dtype} {rule}", x, dtype, u, temperature=temperature, **rule)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_vocabulary(dtype):
    """2^19 tokens.  Weights are off by 2^-44 and 2^-44.6 of themselves, at most 1 each, so a sum of V of them by V (2^-44 + 2^-44.6), relative to the row's total."""
    import torch
    from paper_2105_04779_amd import el_attn
    V = 1 << 19
    g = np.random.default_rng(41)
    x, u = wl.round_to_storage(g.standard_normal((4, V), dtype=np.float32) * np.float32(2), dtype), g.random(4, dtype=np.float32)
    x[3, g.random(V) < 0.5] = -np.inf
    full = lambda v, t: np.full(4, v, t)
    for temperature, k, p, q in ((1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.5, 300000, 0.99, 0.0), (1.0, 50, 1.0, 0.0), (1.5, 0, 1.0, 0.01)):
        want, want_logprob, margin = oracle.sample_tokens_reference(x, u, full(temperature, np.float32), full(k, np.int32), full(p, np.float32), full(q, np.float32))
        tokens, logprob = el_attn.sample_tokens(to_device(x, dtype), torch.from_numpy(u).cuda(), temperature=temperature, top_k=k, top_p=p, min_p=q)
        torch.cuda.synchronize()
        z = (x - x.max(1, keepdims=True)).astype(np.float64) / temperature
        n = min(k, V) if k else V
        off = V * (2.0 ** -44 + 2.0 ** -44.6) / np.sort(np.exp(z), 1)[:, V - n:].sum(1) / p
        assert (margin > off).all(), (margin, off)
        assert np.array_equal(tokens.cpu().numpy(), want), (temperature, k, p, q)
        err = np.abs(logprob.cpu().numpy() - want_logprob) / (2.0 ** -24 * np.abs(want_logprob) + off)
        record(f"vocabulary 2^19 {dtype} T {temperature} k {k} p {p} min-p {q}: {err.max():.3f} of the bound")
        assert err.max() <= 1.0
