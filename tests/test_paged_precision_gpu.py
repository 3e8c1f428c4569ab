"""How precise attention over pages is where every product is exact (small whole numbers), so that only what follows them errs.

u = 2^-24 (half a step of fp32, relative).  Scores lie at most A below the largest.  Their distance to it is formed in one rounding (u A),
with a factor that is rounded twice (1.3 u A); an exponential is good to 2 u; a tile with a larger maximum, or the join of two wavefronts, scales
what is there once more (u A + 2 u, at most twice for two tiles).  Together D = 4.3 u A + 6 u, whatever the size of the scores.  The output is off by
2 D, by the sums (n / 16 + 64 roundings each), by the parts that a probability is split into (2^-24 of it; in fp16 also 2^-40 of the largest: half
the smallest step of fp16, 2^-25, at a scale of 2^15) and by half a step.
"""
import numpy as np
import pytest

import oracle
from helpers import record, to_device
from test_paged_gpu import HALF_STEP, SMALLEST, Case, _host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _whole_numbers(dtype, lengths, heads=4, d=64, seed=95):
    """A case with queries and keys of whole numbers up to 3."""
    c = Case(seed, dtype, len(lengths), 1, heads, heads, d, 16, lengths)
    g = np.random.default_rng(seed)
    c.q = g.integers(-3, 4, c.q.shape).astype(np.float32)
    c.K = np.where(np.isnan(c.K), c.K, g.integers(-3, 4, c.K.shape)).astype(np.float32)
    return c


def _put(c):
    c.q_d = to_device(c.q, c.dtype)
    c.cache.K.copy_(to_device(c.K, c.dtype))
    c.cache.V.copy_(to_device(c.V, c.dtype))


def _compare(tag, c, A, scale, largest_only=0.0, **rule):
    """Against fp64, every output and log-sum-exp within its bound; scale in fp32."""
    out, lse = c.cache.attend_segment(c.q_d, c.table_d, c.lengths_d, scale=scale, **rule)
    ref, ref_lse, info = oracle.paged_attend_reference(c.K, c.V, c.table, c.lengths, c.q, scale=float(np.float32(scale)), **rule)
    out, lse = _host(out).reshape(ref.shape), _host(lse).reshape(ref_lse.shape)
    D, sums = 4.3 * U * A + 6 * U, (info["n"] / 16 + 64) * U
    bound = (2 * D + 2 * sums + 2.0 ** -24)[..., None] * info["spread"] + largest_only
    bound = bound + HALF_STEP["f32"] * (np.abs(ref) + bound) + 1e-37
    worst = float((np.abs(out - ref) / bound).max())
    err = float((np.abs(lse - ref_lse) / (D + sums + 2 * U * np.abs(ref_lse) + 1e-37)).max())
    record(f"{tag}: {worst:.3f} of the bound, lse {err:.3f} of its")
    assert worst <= 1 and err <= 1, f"{tag}: {worst:.3f} of the bound, lse {err:.3f} of its"


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("scale", [0.125, 0.1])
@pytest.mark.parametrize("side", [1, -1])
def test_scores_far_from_zero_keep_their_distances(dtype, scale, side):
    """Thousands that all scores have in common (keys with a large component along the query) take no digits from their differences."""
    c = _whole_numbers(dtype, [33, 64, 40, 57, 48, 64])
    c.q[:] = 16.0
    c.K[:] = np.where(np.isnan(c.K), c.K, 32.0 * side)
    g = np.random.default_rng(96)
    c.K[..., 0] = np.where(np.isnan(c.K[..., 0]), np.nan, 32.0 * side + g.integers(-1, 2, c.K.shape[:3]))       # scores apart by 16 scale
    c.K[..., 1] = np.where(np.isnan(c.K[..., 1]), np.nan, 32.0 * side + g.integers(0, 2, c.K.shape[:3]))
    _put(c)
    _compare(f"far scores {dtype} scale {scale} side {side}", c, 3 * 16 * scale, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("scale", [0.1, 0.013])
def test_log_sum_exp_of_one_position_is_its_score(dtype, scale):
    """2 u of the score, and what the exponential and the logarithm of nearly 1 are off by: 2 u each, and 2 u for their product with ln 2."""
    c = _whole_numbers(dtype, [1] * 60, heads=8)
    _put(c)
    _, lse = c.cache.attend_segment(c.q_d, c.table_d, c.lengths_d, scale=scale)
    _, ref, _ = oracle.paged_attend_reference(c.K, c.V, c.table, c.lengths, c.q, scale=float(np.float32(scale)))
    err = float((np.abs(_host(lse).reshape(ref.shape) - ref) / (2 * U * np.abs(ref) + 6 * U)).max())
    record(f"lse of one position {dtype} scale {scale}: {err:.3f} of the bound")
    assert err <= 1


def test_small_probabilities_in_fp16():
    """One position holds nearly all, with a value of 0; what the others, 2^-26 to 2^-31 of it each, add up to is the output."""
    c = _whole_numbers("f16", [33, 64, 40, 57, 48, 64] * 10)
    c.V = np.abs(c.V)
    n = np.asarray(c.lengths)
    c.q[:] = 1.0
    c.K[:] = np.where(np.isnan(c.K), c.K, 0.0)
    g = np.random.default_rng(97)
    low = g.integers(180, 215, (60, 4))                              # a tenth of each: 18 to 21.4 in natural units
    for b in range(60):
        for t in range(n[b]):
            page, at = int(c.table[b, t // 16]), t % 16
            c.K[page, at, :, 0] = 0 if t == n[b] // 2 else -low[b]
            if t == n[b] // 2:
                c.V[page, at] = 0
    _put(c)
    every = np.stack([c.V[c.table[b, :-(-n[b] // 16)]].reshape(-1, 4, 64)[:n[b]].sum(0) for b in range(60)])[:, None]
    _compare("small probabilities f16", c, 21.5, 0.1, largest_only=2.0 ** -40 * every)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_products_of_fp32_are_summed_in_four_parts(d):
    """One product of 2^24 and d - 1 of a quarter.  An instruction adds four products to one of four sums; at 2^24, where fp32 has steps of 2, it may lose
    all of the 1 that it adds.  One of the sums holds the large product: d / 16 instructions.  Joining the sums rounds three times by 1 at most, the
    log-sum-exp of the one position by 2 (2 u of 2^24).  (One sum of all would lose d / 4 - 1.)"""
    c = Case(99, "f32", 5, 1, 4, 4, d, 16, [1, 1, 1, 1, 1])
    c.q[:] = 0.5
    c.K[:] = np.where(np.isnan(c.K), c.K, 0.5)
    for b in range(5):                                               # the large one in another place for each
        c.q[b, ..., 3 * b], c.K[c.table[b, 0], 0, :, 3 * b] = 4096.0, 4096.0
    _put(c)
    out, lse = c.cache.attend_segment(c.q_d, c.table_d, c.lengths_d, scale=1.0)
    err = np.abs(_host(lse).astype(np.float64) - (2.0 ** 24 + (d - 1) / 4)).max()
    record(f"products of fp32 d {d}: {err:.1f} of {d / 16 + 5:.1f}")
    assert err <= d / 16 + 5
    assert np.array_equal(_host(out).reshape(5, 4, d), np.stack([c.V[c.table[b, 0], 0] for b in range(5)]))
