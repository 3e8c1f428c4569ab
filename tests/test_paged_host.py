"""The paged cache and the token scores without a GPU: refusals before any device work, and the references that the GPU
tests compare with, pinned by closed forms and by torch."""
import ctypes

import numpy as np
import pytest
import torch

import oracle


@pytest.fixture(scope="module")
def ea():
    from paper_2105_04779_amd import el_attn
    return el_attn


P = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(8)]          # never dereferenced
ODD = ctypes.c_void_p(0x100004)


def _pages(ea, **kw):
    base = dict(K=P[0], V=P[1], page_stride=16 * 8 * 128, position_stride=8 * 128, head_stride=128, pages=40, page_size=16,
                kv_heads=8, d_head=128, dtype=ea.EL_BF16)
    base.update(kw)
    return ea.ElAttnPages(**base)


def _calls(ea):
    """name -> call(cache, **changes) with operands that only a device is missing for."""
    def attend(cache, rule=None, **kw):
        a = dict(table=P[2], table_stride=10, table_pages=10, lengths=P[3], queries=P[4], query_stride=32 * 128, heads=32,
                 rule=rule or ea.ElAttnScoreRule(0.1, 0.0, 0, None), out=P[5], out_dtype=ea.EL_BF16, lse=None, B=4, beam=1, n=160,
                 workspace=P[6], workspace_bytes=1 << 40)
        a.update(kw)
        return ea.el_attn_paged_attend(cache, **a)

    def append(cache, **kw):
        a = dict(table=P[2], table_stride=10, table_pages=10, lengths=P[3], counts=None, K_new=P[4], V_new=P[5],
                 batch_stride=3 * 1024, token_stride=1024, B=4, T=3)
        a.update(kw)
        return ea.el_attn_paged_append(cache, **a)

    def copy(cache, **kw):
        a = dict(src=P[2], dst=P[3], counts=None, pairs=5)
        a.update(kw)
        return ea.el_attn_paged_copy(cache, **a)
    return {"attend": attend, "append": append, "copy": copy}


@pytest.mark.parametrize("name", ["attend", "append", "copy"])
def test_a_cache_that_is_none_is_refused(ea, name):
    call, I, U = _calls(ea)[name], ea.EL_ERR_INVALID_ARG, ea.EL_ERR_UNSUPPORTED
    for bad in (dict(K=None), dict(V=None), dict(pages=0), dict(page_size=0), dict(kv_heads=0), dict(d_head=0), dict(K=ODD),
                dict(page_stride=-16 * 8 * 128), dict(position_stride=8 * 128 + 4),
                dict(page_stride=16 * 8 * 128 - 8), dict(position_stride=7 * 128), dict(head_stride=0), dict(head_stride=120),
                dict(page_stride=1 << 45), dict(page_stride=1 << 43, pages=1 << 20)):
        assert call(_pages(ea, **bad)) == I, bad
    for bad in (dict(dtype=7), dict(d_head=264), dict(d_head=4, head_stride=128), dict(dtype=ea.EL_F32, d_head=6)):
        assert call(_pages(ea, **bad)) == U, bad


def test_attend_refuses_bad_operands(ea):
    call, I, U = _calls(ea)["attend"], ea.EL_ERR_INVALID_ARG, ea.EL_ERR_UNSUPPORTED
    c = _pages(ea)
    for bad in (dict(table=None), dict(table=ctypes.c_void_p(0x100002)), dict(table_stride=9), dict(table_pages=0), dict(B=0), dict(beam=0),
                dict(n=0), dict(n=161), dict(queries=None), dict(queries=ODD), dict(out=None), dict(out=ODD), dict(heads=0), dict(heads=12),
                dict(query_stride=32 * 128 - 8), dict(query_stride=32 * 128 + 4), dict(lengths=ctypes.c_void_p(0x100002)),
                dict(lse=ctypes.c_void_p(0x100001)), dict(B=1 << 20, beam=1 << 8)):
        assert call(c, **bad) == I, bad
    for out_dtype in (ea.EL_F16, 9):
        assert call(c, out_dtype=out_dtype) == U
    inf, nan = float("inf"), float("nan")
    for rule in ((inf, 0, 0, None), (nan, 0, 0, None), (0.1, -1.0, 0, None), (0.1, inf, 0, None), (0.1, nan, 0, None), (0.1, 0, -1, None), (1.0, 1e-44, 0, None), (3e38, 0, 0, None),
                 (0.1, 0, 0, ctypes.c_void_p(0x100002))):
        assert call(c, rule=ea.ElAttnScoreRule(*rule)) == I, rule
    need = ea.el_attn_paged_workspace_bytes(c, 32, 4, 1, 160)
    if need:
        assert call(c, workspace_bytes=need - 1) == ea.EL_ERR_WORKSPACE
        assert call(c, workspace=None) == ea.EL_ERR_WORKSPACE
        assert call(c, workspace=ctypes.c_void_p(0x100008)) == I
    assert ea.el_attn_paged_workspace_bytes(_pages(ea, pages=0), 32, 4, 1, 160) == 0


def test_attend_refuses_an_output_among_the_queries(ea):
    call, c = _calls(ea)["attend"], _pages(ea)
    row, at = 32 * 128 * 2, 0x40000000                               # bytes of a row of bf16 heads; four rows
    none = dict(table_stride=200, table_pages=200, n=3200, workspace_bytes=0, workspace=None)      # (refused behind the check: nothing is launched)
    assert ea.el_attn_paged_workspace_bytes(c, 32, 4, 1, 3200) > 0
    for queries, out in ((at, at), (at, at + 4 * row - 16), (at + 4 * row - 16, at)):
        assert call(c, queries=ctypes.c_void_p(queries), out=ctypes.c_void_p(out), **none) == ea.EL_ERR_INVALID_ARG
    for queries, out in ((at, at + 4 * row), (at + 4 * row, at)):
        assert call(c, queries=ctypes.c_void_p(queries), out=ctypes.c_void_p(out), **none) == ea.EL_ERR_WORKSPACE
    # rows further apart, and an output of fp32
    assert call(c, queries=ctypes.c_void_p(at), query_stride=row, out=ctypes.c_void_p(at + 5 * row), **none) == ea.EL_ERR_INVALID_ARG
    assert call(c, queries=ctypes.c_void_p(at + 5 * row), out=ctypes.c_void_p(at), out_dtype=ea.EL_F32, **none) == ea.EL_ERR_INVALID_ARG


def test_append_and_copy_refuse_bad_operands(ea):
    I, c = ea.EL_ERR_INVALID_ARG, _pages(ea)
    call = _calls(ea)["append"]
    for bad in (dict(table=None), dict(table_stride=9), dict(lengths=None), dict(K_new=None), dict(V_new=None), dict(K_new=ODD), dict(T=0),
                dict(B=0), dict(B=70000), dict(token_stride=1016), dict(token_stride=1028), dict(batch_stride=1016),
                dict(counts=ctypes.c_void_p(0x100002))):
        assert call(c, **bad) == I, bad
    call = _calls(ea)["copy"]
    for bad in (dict(src=None), dict(dst=None), dict(pairs=0), dict(src=ctypes.c_void_p(0x100002)), dict(counts=ctypes.c_void_p(0x100001))):
        assert call(c, **bad) == I, bad


def test_scores_refuse_bad_operands(ea):
    I = ea.EL_ERR_INVALID_ARG

    def call(**kw):
        a = dict(dtype=ea.EL_BF16, logits=P[0], row_stride=1000, rows=4, vocab=999, tokens=P[1], logprob=P[2], entropy=P[3], k=5,
                 top_logprob=P[4], top_index=P[5], workspace=P[6], workspace_bytes=1 << 40)
        a.update(kw)
        return ea.el_attn_score_tokens(**a)
    for bad in (dict(logits=None), dict(rows=0), dict(vocab=0), dict(k=-1), dict(k=ea.el_attn_max_alternatives() + 1), dict(tokens=None),
                dict(top_logprob=None), dict(top_index=None), dict(row_stride=998), dict(logits=ctypes.c_void_p(0x100001)),
                dict(tokens=ctypes.c_void_p(0x100002)), dict(entropy=ctypes.c_void_p(0x100002))):
        assert call(**bad) == I, bad
    assert call(dtype=4) == ea.EL_ERR_UNSUPPORTED
    need = ea.el_attn_score_workspace_bytes(4, 999, 5)
    if need:
        assert call(workspace_bytes=need - 1) == ea.EL_ERR_WORKSPACE and call(workspace=None) == ea.EL_ERR_WORKSPACE
    assert ea.el_attn_max_alternatives() >= 32
    for none in ((0, 9, 1), (1, 0, 1), (1, 9, -1), (1, 9, 1000)):
        assert ea.el_attn_score_workspace_bytes(*none) == 0


def test_binding_refuses_what_is_not_on_the_device(ea):
    K = torch.zeros((4, 16, 2, 64))
    with pytest.raises(ValueError):
        ea.PagedCache(K, K.clone())
    with pytest.raises(ValueError):
        ea.score_tokens(torch.zeros((2, 9)))


# ---- pins of the references ----------------------------------------------------------------------------------------------
def _random_cache(g, pages=9, page=5, kv=2, d=8):
    return g.standard_normal((pages, page, kv, d)), g.standard_normal((pages, page, kv, d))


def test_attend_reference_is_torchs_attention():
    g = np.random.default_rng(3)
    K, V = _random_cache(g)
    table, lengths = np.array([[7, 2, 0], [3, 8, 1]]), np.array([13, 5])
    q = g.standard_normal((2, 3, 4, 8))
    out, lse, _ = oracle.paged_attend_reference(K, V, table, lengths, q, scale=8 ** -0.5)
    for b in range(2):
        k = torch.from_numpy(K[table[b]].reshape(15, 2, 8)[:lengths[b]]).permute(1, 0, 2).repeat_interleave(2, 0)
        v = torch.from_numpy(V[table[b]].reshape(15, 2, 8)[:lengths[b]]).permute(1, 0, 2).repeat_interleave(2, 0)
        qb = torch.from_numpy(q[b]).permute(1, 0, 2)
        want = torch.nn.functional.scaled_dot_product_attention(qb, k, v).permute(1, 0, 2)
        assert np.abs(out[b] - want.numpy()).max() < 1e-12
        assert np.abs(lse[b].T - torch.logsumexp(qb @ k.transpose(1, 2) * 8 ** -0.5, 2).numpy()).max() < 1e-12


def test_attend_reference_rules_and_empty_rows():
    g = np.random.default_rng(4)
    K, V = _random_cache(g, kv=1)
    table, q = np.array([[4, -1, 6]]), g.standard_normal((1, 1, 1, 8))
    rule = dict(scale=1.0)
    # one position left: its value, and its score as the log-sum-exp; distance of the newest position is 0
    out, lse, _ = oracle.paged_attend_reference(K, V, table, [3], q, window=1, softcap=2.0, slopes=[5.0], **rule)
    assert np.allclose(out[0, 0, 0], V[4, 2, 0]) and np.isclose(lse[0, 0, 0], 2 * np.tanh(K[4, 2, 0] @ q[0, 0, 0] / 2))
    # a bias by distance shifts the log-sum-exp of a single older position
    out, lse, _ = oracle.paged_attend_reference(K, V, np.array([[4, -1, -1]]), [15], q, window=11, slopes=[0.25], **rule)
    assert np.allclose(out[0, 0, 0], V[4, 4, 0]) and np.isclose(lse[0, 0, 0], K[4, 4, 0] @ q[0, 0, 0] - 0.25 * 10)
    # absent pages, length 0, windows inside an absent page
    for kw, length in ((dict(), 0), (dict(window=3), 10)):
        out, lse, _ = oracle.paged_attend_reference(K, V, table, [length], q, **kw, **rule)
        assert not out.any() and lse[0, 0, 0] == -np.inf
    # what no position names does not matter
    K2, V2 = K.copy(), V.copy()
    K2[[0, 1, 2, 3, 5, 7, 8]] = np.nan
    V2[6, 1:] = np.inf
    a, b = (oracle.paged_attend_reference(k, v, table, [11], q, **rule)[0] for k, v in ((K, V), (K2, V2)))
    assert np.array_equal(a, b)


def test_append_and_copy_references():
    g = np.random.default_rng(5)
    K, V = _random_cache(g)
    kn, vn = g.standard_normal((2, 4, 2, 8)), g.standard_normal((2, 4, 2, 8))
    table = np.array([[7, 2], [3, -1]])
    K2, V2 = oracle.paged_append_reference(K, V, table, [7, 6], [4, 2], kn, vn)
    assert np.array_equal(K2[7, 3:], kn[0, :2]) and np.array_equal(V2[2, :2], vn[0, 2:]) and np.array_equal(K2[3, 4], kn[1, 0])
    untouched = np.ones((9, 5), bool)
    untouched[7, 3:] = untouched[2, :2] = untouched[3, 4] = False
    assert np.array_equal(K2[untouched], K[untouched]) and np.array_equal(V2[untouched], V[untouched])
    K3, V3 = oracle.paged_copy_reference(K, V, [1, 1, 9, 0], [4, 5, 6, -1], [2, 9, 3, 3])
    assert np.array_equal(K3[4, :2], K[1, :2]) and np.array_equal(K3[4, 2:], K[4, 2:]) and np.array_equal(V3[5], V[1])
    assert np.array_equal(K3[[6, 0, 8]], K[[6, 0, 8]])


def test_scores_reference_is_torchs():
    g = np.random.default_rng(6)
    x = g.standard_normal((5, 37)) * 3
    x[1, 5:] = -np.inf
    x[2, [3, 9, 20]] = 50.0
    t = torch.from_numpy(x)
    logp = torch.log_softmax(t, 1)
    tokens = np.array([0, 36, 9, -1, 40])
    logprob, entropy, top, index, _ = oracle.score_tokens_reference(x, tokens, 7)
    assert np.allclose(logprob[[0, 2]], logp[[0, 2], [0, 9]].numpy()) and logprob[1] == -np.inf and logprob[3] == 0 and np.isnan(logprob[4])
    want = torch.distributions.Categorical(logits=t[[0, 2, 3, 4]]).entropy().numpy()
    assert np.allclose(entropy[[0, 2, 3, 4]], want, atol=1e-9)
    assert list(index[2][:3]) == [3, 9, 20] and list(index[1][5:]) == [-1, -1] and top[1, 6] == -np.inf
    assert np.allclose(top[0], torch.sort(logp[0], descending=True)[0][:7].numpy())
    uniform = oracle.score_tokens_reference(np.full((1, 64), 2.5), None, 3)
    assert np.isclose(uniform[1][0], np.log(64)) and list(uniform[3][0]) == [0, 1, 2]
    lowest = oracle.score_tokens_reference(np.full((2, 64), [[-3.4e38], [3.4e38]]), [5, 9], 2)      # whatever size the logits have
    assert np.allclose(lowest[0], -np.log(64)) and np.allclose(lowest[1], np.log(64)) and np.allclose(lowest[2], -np.log(64))
    none = oracle.score_tokens_reference(np.full((1, 8), -np.inf), [3], 2)
    assert none[0][0] == -np.inf and none[1][0] == 0 and list(none[3][0]) == [-1, -1]
    assert np.isnan(oracle.score_tokens_reference(np.array([[1.0, np.nan, 3.0]]), [0], 2)[1][0])
