"""Calls of the paged cache and the token scores at the edges of what they take: no work, operands that ask for a derivative,
values that are not finite."""
import numpy as np
import pytest

import oracle
from paper_2105_04779_amd import workloads as wl
from helpers import to_device
from test_paged_gpu import Case, _host

pytestmark = pytest.mark.gpu


def test_no_work_is_no_error():
    """A step without forks, without new tokens, of no sequence or no beam, scores of no row: nothing moves, empty results."""
    import torch
    from paper_2105_04779_amd import el_attn
    c = Case(90, "bf16", 2, 2, 4, 2, 64, 16, [20, 33])
    K, V = c.cache.K.clone(), c.cache.V.clone()
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    c.cache.copy_pages(none, none)
    c.cache.copy_pages(none, none, none)
    c.cache.append(c.q_d[:, :0, :2], c.q_d[:, :0, :2], c.table_d, c.lengths_d)
    c.cache.append(c.q_d[:0, :, :2], c.q_d[:0, :, :2], c.table_d[:0], none, none)
    for q, table, lengths in ((c.q_d[:0], c.table_d[:0], none), (c.q_d[:0], c.table_d[:0], None), (c.q_d[:, :0], c.table_d, c.lengths_d)):
        rows = q.shape[0] * q.shape[1]
        out = c.cache.attend(q, table, lengths, out_dtype="f32")
        assert out.shape == q.shape and out.dtype == torch.float32
        assert c.cache.attend(q, table, lengths, out=torch.empty_like(q)).shape == q.shape
        A, lse = c.cache.attend_segment(q, table, lengths, window=3)
        assert A.shape == (rows, 4 * 64) and lse.shape == (rows, 4)
    logprob, entropy, top, index = el_attn.score_tokens(torch.zeros((0, 99), device="cuda"), none, k=5)
    assert logprob.shape == entropy.shape == (0,) and top.shape == index.shape == (0, 5) and index.dtype == torch.int32
    assert el_attn.score_tokens(torch.zeros((0, 99), device="cuda"))[0] is None
    torch.cuda.synchronize()
    assert torch.equal(K.nan_to_num(5.0), c.cache.K.nan_to_num(5.0)) and torch.equal(V.nan_to_num(5.0), c.cache.V.nan_to_num(5.0))
    # the checks are those of every call
    for call in (lambda: c.cache.copy_pages(none, none.long()), lambda: c.cache.attend(c.q_d[:0], c.table_d, none), lambda: c.cache.attend(c.q_d[:0].float(), c.table_d[:0], none),
                 lambda: c.cache.append(c.q_d[:0, :, :2], c.q_d[:0, :, :2], c.table_d[:0], none.long()), lambda: el_attn.score_tokens(torch.zeros((0, 99), device="cuda"), k=65)):
        with pytest.raises(ValueError):
            call()
            pytest.fail("taken")


def test_a_tangent_is_refused():
    """Forward-mode differentiation: a result without the tangent would be wrong in silence."""
    import torch
    import torch.autograd.forward_ad as fw
    from paper_2105_04779_amd import el_attn
    c = Case(91, "f32", 2, 2, 4, 2, 64, 16, [20, 33])
    slopes, logits, new = torch.ones(4, device="cuda"), torch.randn((3, 50), device="cuda"), c.q_d[:, :, :2]
    with fw.dual_level():
        dual = lambda t: fw.make_dual(t, torch.ones_like(t))
        for call in (lambda: c.cache.attend(dual(c.q_d), c.table_d, c.lengths_d), lambda: c.cache.attend_segment(dual(c.q_d), c.table_d, c.lengths_d),
                     lambda: c.cache.attend(c.q_d, c.table_d, c.lengths_d, slopes=dual(slopes)),
                     lambda: c.cache.attend(c.q_d, c.table_d, c.lengths_d, out=dual(torch.empty_like(c.q_d))),
                     lambda: c.cache.append(dual(new), new, c.table_d, c.lengths_d), lambda: c.cache.append(new, dual(new), c.table_d, c.lengths_d),
                     lambda: el_attn.PagedCache(dual(c.cache.K), c.cache.V), lambda: el_attn.PagedCache(c.cache.K, dual(c.cache.V)),
                     lambda: el_attn.score_tokens(dual(logits))):
            with pytest.raises(ValueError, match="tangent"):
                call()
                pytest.fail("taken")
        # operands without one are taken there as elsewhere
        a = c.cache.attend(c.q_d, c.table_d, c.lengths_d)
    assert torch.equal(a, c.cache.attend(c.q_d, c.table_d, c.lengths_d))


def test_an_output_that_asks_for_a_gradient_is_refused():
    import torch
    c = Case(92, "f32", 2, 1, 4, 2, 64, 16, [20, 33])
    out = torch.empty_like(c.q_d).requires_grad_()
    with pytest.raises(ValueError):
        c.cache.attend(c.q_d, c.table_d, c.lengths_d, out=out)
    with torch.no_grad():
        assert c.cache.attend(c.q_d, c.table_d, c.lengths_d, out=out) is out
    assert torch.equal(out.detach(), c.cache.attend(c.q_d, c.table_d, c.lengths_d))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,n", [(3, 50), (3, 3000)])
def test_values_that_are_not_finite_stay_in_their_column(dtype, B, n):
    """A position that is there passes an infinite or NaN value on to its column, its probability 0 or not (a score of -inf, or one
    that underflows); other columns and other sequences know nothing of it.  A row whose scores are all -inf is 0.  n: a sequence
    taken whole, and cut ones."""
    c = Case(93, dtype, B, 2, 4, 2, 64, 16, [n, n, n - 3])
    c.q = wl.round_to_storage(np.minimum(np.abs(c.q) + np.float32(0.5), np.float32(4.0)), dtype)
    c.q_d = to_device(c.q, dtype)
    K, V = c.cache.K, c.cache.V
    last = int(c.table[0, (n - 1) // 16])                            # the first sequence's newest position, and its very first
    K[last, (n - 1) % 16] = -float("inf")
    c.K[last, (n - 1) % 16] = -np.inf
    V[last, (n - 1) % 16, :, 5] = float("inf")
    V[int(c.table[0, 0]), 0, :, 17] = float("nan")
    K[int(c.table[0, 1]), 2], c.K[int(c.table[0, 1]), 2] = -300.0, -300.0        # scores hundreds below the rest
    V[int(c.table[0, 1]), 2, :, 40] = -float("inf")
    for page in c.table[1]:                                          # the second sequence: no score above -inf, no finite value
        K[int(page)], V[int(page)] = -float("inf"), float("nan")
        c.K[int(page)] = -np.inf
        c.V[int(page)] = 0
    ref, ref_lse, _ = oracle.paged_attend_reference(c.K, c.V, c.table, c.lengths, c.q, scale=0.125)
    A, lse = c.cache.attend_segment(c.q_d, c.table_d, c.lengths_d)
    A, lse = _host(A).reshape(ref.shape), _host(lse).reshape(ref_lse.shape)
    hit = np.zeros(ref.shape, bool)
    hit[0][..., [5, 17, 40]] = True
    assert not np.isfinite(A[hit]).any()
    assert not A[1].any() and np.isneginf(lse[1]).all()
    assert np.abs(A - ref)[~hit].max() < 1e-4 * np.abs(ref).max()
    assert np.abs(lse[[0, 2]] - ref_lse[[0, 2]]).max() < 1e-4 * np.abs(ref_lse[[0, 2]]).max()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_cap_of_any_size(dtype):
    """Beyond the scores' own size a cap changes nothing, up to the largest number there is.  Scores up to 2.5, caps from 1e6: (s / c)^2 / 3 is
    below 2^-40.  Whole numbers: the products are exact.  scale / c loses digits among the subnormal numbers, 2^-150 of 0.1 / 3.4e38 = 2^-131.3 at most: 2^-18.7 of a score."""
    import torch
    c = Case(94, dtype, 3, 1, 4, 4, 64, 16, [33, 64, 40])
    g = np.random.default_rng(94)
    c.q_d.copy_(torch.from_numpy(g.integers(-1, 2, c.q.shape) * (np.arange(64) < 25)))
    c.cache.K.copy_(torch.from_numpy(g.integers(-1, 2, c.K.shape)))
    none, none_lse = (_host(t) for t in c.cache.attend_segment(c.q_d, c.table_d, c.lengths_d, scale=0.1))
    spread = np.nanmax(np.abs(c.V))
    for cap in (1e6, 1e30, 3.0e38, 3.4028234663852886e38):
        A, lse = (_host(t) for t in c.cache.attend_segment(c.q_d, c.table_d, c.lengths_d, scale=0.1, softcap=cap))
        D = 2.5 * (2.0 ** -18.7 if cap > 1e30 else 0.0) + 2.5 * 8 * 2.0 ** -24 + 16 * 2.0 ** -24 + 80 * 2.0 ** -24
        assert np.isfinite(A).all() and np.isfinite(lse).all(), cap
        assert np.abs(A - none).max() <= 4 * D * spread and np.abs(lse - none_lse).max() <= 2 * D, cap
