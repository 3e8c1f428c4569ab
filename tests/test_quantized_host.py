"""The paged cache in 8 bits, the page plan and sampling without a GPU: refusals before any device work, and the references that the GPU
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


P = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(12)]         # never dereferenced
ODD, ODD4 = ctypes.c_void_p(0x100008), ctypes.c_void_p(0x100002)


def _pages(ea, **kw):
    base = dict(K=P[0], V=P[1], K_scale=P[8], V_scale=P[9], page_stride=16 * 8 * 128, position_stride=8 * 128, head_stride=128, pages=40, page_size=16,
                kv_heads=8, d_head=128, block=8, format=ea.EL_E4M3)
    base.update(kw)
    return ea.ElAttnPages8(**base)


def _calls(ea):
    """name -> call(cache, **changes) with operands that only a device is missing for."""
    def attend(cache, rule=None, **kw):
        a = dict(dtype=ea.EL_BF16, table=P[2], table_stride=200, table_pages=200, lengths=P[3], queries=P[4], query_stride=32 * 128, heads=32,
                 rule=rule or ea.ElAttnScoreRule(0.1, 0.0, 0, None), out=P[5], out_dtype=ea.EL_BF16, lse=None, B=4, beam=1, n=3200,
                 workspace=P[6], workspace_bytes=1 << 40)
        a.update(kw)
        return ea.el_attn_quantized_attend(cache, **a)

    def append(cache, **kw):
        a = dict(dtype=ea.EL_BF16, table=P[2], table_stride=10, table_pages=10, lengths=P[3], counts=None, K_new=P[4], V_new=P[5],
                 batch_stride=3 * 1024, token_stride=1024, B=4, T=3)
        a.update(kw)
        return ea.el_attn_quantized_append(cache, **a)

    def copy(cache, **kw):
        a = dict(src=P[2], dst=P[3], counts=None, pairs=5)
        a.update(kw)
        return ea.el_attn_quantized_copy(cache, **a)
    return {"attend": attend, "append": append, "copy": copy}


@pytest.mark.parametrize("name", ["attend", "append", "copy"])
def test_a_cache_that_is_none_is_refused(ea, name):
    call, I, U = _calls(ea)[name], ea.EL_ERR_INVALID_ARG, ea.EL_ERR_UNSUPPORTED
    for bad in (dict(K=None), dict(V=None), dict(K_scale=None), dict(V_scale=None), dict(pages=0), dict(page_size=0), dict(kv_heads=0), dict(d_head=0),
                dict(K=ODD), dict(V_scale=ODD4), dict(page_stride=-16 * 8 * 128), dict(position_stride=8 * 128 + 8), dict(page_stride=16 * 8 * 128 - 16),
                dict(position_stride=7 * 128), dict(head_stride=0), dict(head_stride=112), dict(page_stride=1 << 45), dict(page_stride=1 << 43, pages=1 << 20),
                dict(block=0), dict(block=3), dict(block=32), dict(block=-8)):
        assert call(_pages(ea, **bad)) == I, bad
    for bad in (dict(format=0), dict(format=3), dict(d_head=272), dict(d_head=120), dict(d_head=8), dict(page_size=1 << 17, page_stride=1 << 30, block=8)):
        assert call(_pages(ea, **bad)) == U, bad


def test_attend_refuses_bad_operands(ea):
    call, I, U = _calls(ea)["attend"], ea.EL_ERR_INVALID_ARG, ea.EL_ERR_UNSUPPORTED
    c = _pages(ea)
    for bad in (dict(table=None), dict(table=ODD4), dict(table_stride=199), dict(table_pages=0), dict(B=0), dict(beam=0), dict(n=0), dict(n=3201),
                dict(queries=None), dict(queries=ODD), dict(out=None), dict(out=ODD), dict(heads=0), dict(heads=12), dict(query_stride=32 * 128 - 8),
                dict(query_stride=32 * 128 + 4), dict(lengths=ODD4), dict(lse=ODD4), dict(B=1 << 20, beam=1 << 8), dict(out=P[4])):
        assert call(c, **bad) == I, bad
    for bad in (dict(dtype=3), dict(dtype=-1), dict(out_dtype=ea.EL_F16), dict(out_dtype=9), dict(dtype=ea.EL_F32, out_dtype=ea.EL_BF16)):
        assert call(c, **bad) == U, bad
    inf, nan = float("inf"), float("nan")
    for rule in ((inf, 0, 0, None), (nan, 0, 0, None), (0.1, -1.0, 0, None), (0.1, inf, 0, None), (0.1, 0, -1, None), (1.0, 1e-44, 0, None), (3e38, 0, 0, None),
                 (0.1, 0, 0, ODD4)):
        assert call(c, rule=ea.ElAttnScoreRule(*rule)) == I, rule
    need = ea.el_attn_quantized_workspace_bytes(c, ea.EL_BF16, ea.EL_BF16, 32, 4, 1, 3200)
    assert need > 0
    assert call(c, workspace_bytes=need - 1) == ea.EL_ERR_WORKSPACE and call(c, workspace=None) == ea.EL_ERR_WORKSPACE
    assert call(c, workspace=ODD) == I
    assert ea.el_attn_quantized_workspace_bytes(_pages(ea, pages=0), ea.EL_BF16, ea.EL_BF16, 32, 4, 1, 3200) == 0
    assert ea.el_attn_quantized_workspace_bytes(c, ea.EL_BF16, ea.EL_F16, 32, 4, 1, 3200) == 0


def test_append_and_copy_refuse_bad_operands(ea):
    I, U, c = ea.EL_ERR_INVALID_ARG, ea.EL_ERR_UNSUPPORTED, _pages(ea)
    call = _calls(ea)["append"]
    for bad in (dict(table=None), dict(table_stride=9), dict(lengths=None), dict(K_new=None), dict(V_new=None), dict(K_new=ODD), dict(T=0), dict(B=0),
                dict(B=70000), dict(token_stride=1016), dict(token_stride=1028), dict(batch_stride=1016), dict(counts=ODD4), dict(T=(1 << 23) + 1)):
        assert call(c, **bad) == I, bad
    for bad in (dict(dtype=5), dict(dtype=-1)):
        assert call(c, **bad) == U, bad
    assert call(_pages(ea, block=1, page_size=16), B=65535, T=1 << 20, batch_stride=1 << 31) == U        # a grid beyond 2^31 workgroups
    call = _calls(ea)["copy"]
    for bad in (dict(src=None), dict(dst=None), dict(pairs=0), dict(pairs=(1 << 23) + 1), dict(src=ODD4), dict(counts=ODD4)):
        assert call(c, **bad) == I, bad


def test_append_refuses_what_a_launch_cannot_hold(ea):
    """A workgroup of 256 lanes has four (block, head, K or V): 2^24 workgroups would be 2^32 lanes."""
    call, wide = _calls(ea)["append"], dict(block=1, kv_heads=32, position_stride=32 * 128, page_stride=16 * 32 * 128)
    token = dict(token_stride=32 * 128, batch_stride=1 << 36)
    for B, T in ((1, 1 << 20), (1, (1 << 20) + 1), (3, 1 << 20), (1, 1 << 23)):          # T blocks, 16 T workgroups
        assert call(_pages(ea, **wide), B=B, T=T, **token) == ea.EL_ERR_UNSUPPORTED, (B, T)


def test_plan_refuses_bad_operands(ea):
    I = ea.EL_ERR_INVALID_ARG

    def call(**kw):
        a = dict(table=P[0], table_stride=20, columns=20, lengths=P[1], B_old=5, parents=P[2], counts=P[3], reserved=None, pages=100, page_size=16, B=7, T=3,
                 new_table=P[4], new_lengths=P[5], granted=P[6], slots=P[7], copies=P[8], free_pages=P[9], workspace=P[10], workspace_bytes=1 << 30)
        a.update(kw)
        return ea.el_attn_plan_pages(**a)
    for bad in (dict(table=None), dict(lengths=None), dict(new_table=None), dict(new_lengths=None), dict(granted=None), dict(copies=None), dict(free_pages=None),
                dict(table=ODD4), dict(parents=ODD4), dict(slots=ctypes.c_void_p(0x100004)), dict(columns=0), dict(table_stride=19), dict(B=0), dict(B_old=0),
                dict(B=(1 << 20) + 1), dict(pages=0), dict(pages=(1 << 24) + 1), dict(page_size=0), dict(page_size=1 << 28), dict(T=0), dict(T=(1 << 23) + 1),
                dict(parents=None), dict(table_stride=(1 << 40) + 1), dict(workspace=ODD)):
        assert call(**bad) == I, bad
    need = ea.el_attn_plan_workspace_bytes(7, 100)
    assert need > 0 and call(workspace_bytes=need - 1) == ea.EL_ERR_WORKSPACE and call(workspace=None) == ea.EL_ERR_WORKSPACE
    for none in ((0, 9), (9, 0), ((1 << 20) + 1, 9), (9, (1 << 24) + 1)):
        assert ea.el_attn_plan_workspace_bytes(*none) == 0


def test_sampling_refuses_bad_operands(ea):
    I = ea.EL_ERR_INVALID_ARG
    rule = lambda t=1.0, rt=None, rk=None, rp=None, rm=None: ea.ElAttnSampleRule(t, 0, 1.0, 0.0, rt, rk, rp, rm)

    def call(**kw):
        a = dict(dtype=ea.EL_BF16, logits=P[0], row_stride=1000, rows=4, vocab=999, uniform=P[1], rule=rule(), tokens=P[2], logprob=P[3],
                 workspace=P[4], workspace_bytes=1 << 40)
        a.update(kw)
        return ea.el_attn_sample_tokens(**a)
    for bad in (dict(logits=None), dict(uniform=None), dict(rule=None), dict(tokens=None), dict(rows=0), dict(rows=(1 << 23) + 1), dict(vocab=0), dict(row_stride=998),
                dict(logits=ctypes.c_void_p(0x100001)), dict(uniform=ODD4), dict(tokens=ODD4), dict(logprob=ODD4), dict(rule=rule(-1.0)), dict(rule=rule(float("nan"))),
                dict(rule=rule(float("inf"))), dict(rule=rule(rt=ODD4)), dict(rule=rule(rk=ODD4)), dict(rule=rule(rp=ODD4)), dict(rule=rule(rm=ODD4)),
                dict(row_stride=1 << 44, rows=1 << 20)):
        assert call(**bad) == I, bad
    for bad in (dict(dtype=4), dict(vocab=(1 << 19) + 1, row_stride=1 << 20)):
        assert call(**bad) == ea.EL_ERR_UNSUPPORTED, bad
    need = ea.el_attn_sample_workspace_bytes(ea.EL_BF16, 4, 999)
    if need:
        assert call(workspace_bytes=need - 1) == ea.EL_ERR_WORKSPACE and call(workspace=None) == ea.EL_ERR_WORKSPACE


def test_binding_refuses_what_is_not_on_the_device(ea):
    K, s = torch.zeros((4, 16, 2, 64), dtype=torch.int8), torch.ones((4, 2, 2))
    with pytest.raises(ValueError):
        ea.PagedCache8(K, K.clone(), s, s.clone())
    with pytest.raises(ValueError):
        ea.sample_tokens(torch.zeros((2, 9)), torch.zeros(2))
    with pytest.raises(ValueError):
        ea.plan_pages(torch.zeros((2, 9), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), pages=4, page_size=16)


def test_the_cache_keeps_the_pools_that_it_was_made_of(ea):
    cache = object.__new__(ea.PagedCache8)
    for name in ("K", "V", "K_scale", "V_scale"):
        with pytest.raises(AttributeError):
            setattr(cache, name, torch.zeros((4, 16, 2, 64)))


# ---- pins of the references ----------------------------------------------------------------------------------------------
def test_codes_are_torchs():
    bits = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(oracle.e4m3_values(), bits.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    g = np.random.default_rng(1)
    y = np.concatenate([g.standard_normal(5000) * 10.0 ** g.uniform(-4, 2.6, 5000), oracle.e4m3_values()[np.r_[:127, 128:255]],
                        (oracle.e4m3_values()[:126] + oracle.e4m3_values()[1:127]) / 2, [0.0, -0.0, 448.0, -448.0]]).astype(np.float32)
    y = np.clip(y, -448, 448)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(oracle.nearest_codes(y, "e4m3"), want)
    assert list(oracle.nearest_codes([1e9, -np.inf, np.nan, 449.0], "e4m3")) == [126, 254, 127, 126]
    assert list(oracle.nearest_codes([0.5, 1.5, -2.5, 126.5, 300.0, -np.inf, np.nan], "int8")) == [0, 2, -2, 126, 127, -127, 0]


def test_append_reference():
    f = np.float32
    codes, scale = np.zeros((3, 8, 1, 16), np.int8), np.full((3, 1, 2), np.nan, f)
    new = np.zeros((1, 3, 1, 16), f)
    new[0, 0, 0, 0], new[0, 1, 0, 3], new[0, 2, 0, 15] = 12.7, -254.0, 1.0
    # the first token of a block sets its scale; a larger one doubles it twenty times, and the first is rounded again
    c, s = oracle.quantized_append_reference(codes, scale, np.array([[2]]), [1], [1], new[:, :1], 4, "int8")
    assert np.isclose(s[2, 0, 0], 0.1) and c[2, 0, 0, 0] == 127 and np.isnan(s[2, 0, 1])
    c, s = oracle.quantized_append_reference(c, s, np.array([[2]]), [2], [1], new[:, 1:2], 4, "int8")
    assert s[2, 0, 0] == 2 and c[2, 0, 0, 0] == 6 and c[2, 1, 0, 3] == -127
    c, s = oracle.quantized_append_reference(c, s, np.array([[2]]), [3], [1], new[:, 2:3], 4, "int8")
    assert s[2, 0, 0] == 2 and c[2, 2, 0, 15] == 0                             # 0.5 to the even code
    # all at once: rounded once
    c1, s1 = oracle.quantized_append_reference(codes, scale, np.array([[2]]), [3], None, new, 4, "int8")
    assert np.array_equal(c1[2, :3], c[2, :3]) and s1[2, 0, 0] == 2
    # a block that a sequence begins anew forgets what it held; negative positions, positions behind the table and absent pages are dropped
    c2, s2 = oracle.quantized_append_reference(c, s, np.array([[2]]), [1], [1], new[:, :1], 4, "int8")
    assert np.isclose(s2[2, 0, 0], 0.1)
    for table, lengths in (([[2]], [0]), ([[2]], [9]), ([[-1]], [3]), ([[3]], [3])):
        c3, s3 = oracle.quantized_append_reference(c, s, np.array(table), lengths, [1], new[:, :1], 4, "int8")
        assert np.array_equal(c3, c) and np.array_equal(s3, s, equal_nan=True)


def test_plan_reference():
    table, lengths = np.array([[5, 6, -1], [7, -1, -1]]), np.array([6, 4])
    # the one goes on in its last page, the other needs a new one: the lowest that nobody names
    p = oracle.plan_pages_reference(table, lengths, None, None, None, 9, 4, 1)
    assert p["table"].tolist() == [[5, 6, -1], [7, 0, -1]] and p["lengths"].tolist() == [7, 5] and p["slots"].tolist() == [[26], [0]] and p["free"] == 5
    assert (p["copies"][:2] == -1).all()
    # two go on from the first, none from the second, whose page is free again: the first keeps the partly filled page, the second gets a copy
    p = oracle.plan_pages_reference(table, lengths, None, [0, 0], None, 9, 4, 1)
    assert p["table"].tolist() == [[5, 6, -1], [5, 0, -1]] and p["copies"].T.tolist() == [[-1, -1, 0], [6, 0, 2]] and p["free"] == 6
    # not enough pages: the first are served
    p = oracle.plan_pages_reference(table, lengths, [1, 1, 9], [0, 1, -1], [0, 1, 1, 1, 1, 0, 0, 0, 0], 9, 4, 9)
    assert p["granted"].tolist() == [1, 1, 0] and p["table"][2].tolist() == [-1] * 3 and p["free"] == 1
    # a sequence that writes nothing does not hold a page against one that does, unless it has more of it
    p = oracle.plan_pages_reference(np.array([[1], [1]]), [2, 3], [1, 0], None, None, 4, 4, 1)
    assert p["table"].tolist() == [[0], [1]] and p["copies"][:, 0].tolist() == [1, 0, 2]
    p = oracle.plan_pages_reference(np.array([[1], [1]]), [3, 3], [0, 1], None, None, 4, 4, 1)
    assert p["table"].tolist() == [[1], [1]] and p["slots"].tolist() == [[-1], [7]]


def test_sampling_reference():
    g = np.random.default_rng(2)
    x = np.tile(g.standard_normal((1, 50)) * 2, (4000, 1))
    u = (np.arange(4000) + 0.5) / 4000
    one = np.ones(4000)
    tokens, logprob, _ = oracle.sample_tokens_reference(x, u, 0.7 * one, 0 * one, one, 0 * one)
    p = torch.softmax(torch.from_numpy(x[0]) / 0.7, 0).numpy()
    assert np.abs(np.bincount(tokens, minlength=50) / 4000 - p).max() <= 1 / 4000 and np.allclose(logprob, np.log(p[tokens]))
    order = np.argsort(-p)
    assert set(oracle.sample_tokens_reference(x, u, 0.7 * one, 5 * one, one, 0 * one)[0]) == set(order[:5])
    n = int(np.searchsorted(np.cumsum(p[order]), 0.6)) + 1
    assert set(oracle.sample_tokens_reference(x, u, 0.7 * one, 0 * one, 0.6 * one, 0 * one)[0]) == set(order[:n])
    assert set(oracle.sample_tokens_reference(x, u, 0.7 * one, 0 * one, one, 0.1 * one)[0]) == set(np.nonzero(p >= 0.1 * p.max())[0])
    # top-p of what top-k left
    k3 = p[order[:3]] / p[order[:3]].sum()
    n = int(np.searchsorted(np.cumsum(k3), k3[0] + 0.5 * k3[1])) + 1
    both = oracle.sample_tokens_reference(x, u, 0.7 * one, 3 * one, (k3[0] + 0.5 * k3[1]) * one, 0 * one)[0]
    assert n == 2 and set(both) == set(order[:2])
    tokens, logprob, _ = oracle.sample_tokens_reference(np.array([[1.0, 3, 3, 2], [-np.inf] * 4, [0, np.nan, 0, 0]]), [0.9] * 3, [0.0] * 3, [0] * 3, [1.0] * 3, [0.0] * 3)
    assert tokens.tolist() == [1, -1, -1] and logprob[0] == 0 and logprob[1] == -np.inf and np.isnan(logprob[2])
