"""The page plan of a cache in 8 bits without a GPU: what a shared page that is written costs those that share it, and the refusals of the call."""
import ctypes

import numpy as np
import pytest

import oracle


@pytest.fixture(scope="module")
def ea():
    from paper_2105_04779_amd import el_attn
    return el_attn


def _fork(fmt, exclusive, pages, counts=(1, 0), T=1):
    """Two sequences share 5 positions of a page of 8; those that `counts` names write, a token 170 times as large as what is there.
    (plan, the second sequence's values before and after)"""
    g = np.random.default_rng(3)
    table, lengths, kv, d, block = np.array([[2, -1], [2, -1]]), np.array([5, 5]), 2, 16, 8
    codes, scale = np.zeros((pages, 8, kv, d), np.int8 if fmt == "int8" else np.uint8), np.ones((pages, kv, 1), np.float32)
    old = g.standard_normal((1, 5, kv, d)).astype(np.float32)
    codes, scale = oracle.quantized_append_reference(codes, scale, table[:1], [5], None, old, block, fmt)

    def values(table, codes, scale):
        page = table[1, 0]
        return oracle.quantized_values(codes[page, :5], fmt) * scale[page, :, 0].astype(np.float64)[None, :, None]
    before = values(table, codes, scale)
    plan = oracle.plan_pages_reference(table, lengths, np.array(counts), None, None, pages, 8, T, exclusive=exclusive)
    codes, scale = oracle.quantized_copy_reference(codes, scale, *plan["copies"], block)
    new = np.full((2, T, kv, d), 400, np.float32)
    codes, scale = oracle.quantized_append_reference(codes, scale, plan["table"], plan["lengths"], plan["granted"], new, block, fmt)
    return plan, before, values(plan["table"], codes, scale)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_write_leaves_those_that_share_and_do_not_write_what_they_have(fmt):
    plan, before, after = _fork(fmt, True, 4)
    assert plan["granted"].tolist() == [1, 0] and plan["copies"].T.tolist() == [[2, 0, 5], [-1, -1, 0]] and plan["table"][:, 0].tolist() == [0, 2] and plan["free"] == 2
    assert np.array_equal(before, after)
    # (the rule for 16 bits, where a write touches no position but its own, keeps the page for the writer)
    plan, before, after = _fork(fmt, False, 4)
    assert (plan["copies"][0] == -1).all() and not np.array_equal(before, after)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_without_a_page_for_the_copy_nothing_is_granted(fmt):
    plan, before, after = _fork(fmt, True, 3, counts=(1, 1))
    # two pages left: one copy each, and the page that both had is named by none
    assert plan["granted"].tolist() == [1, 1] and plan["table"][:, 0].tolist() == [0, 1] and plan["free"] == 0
    plan, before, after = _fork(fmt, True, 3, counts=(4, 1), T=4)
    # the first needs two pages, the second then finds none
    assert plan["granted"].tolist() == [4, 0] and plan["table"].tolist() == [[0, 1], [2, -1]]
    assert np.array_equal(before, after)


def test_who_names_a_page():
    plan = lambda table, lengths, counts, **kw: oracle.plan_pages_reference(np.array(table), np.array(lengths), np.array(counts), None, kw.get("reserved"), 6, 4, 1, exclusive=True)
    # alone: kept; a reader of fewer positions, or the same page twice in one row: copied; reserved: copied
    assert plan([[1, 2]], [6], [1])["copies"].T.tolist() == [[-1, -1, 0]]
    assert plan([[1, 2], [2, -1]], [6, 1], [1, 0])["copies"].T.tolist() == [[2, 0, 2], [-1, -1, 0]]
    assert plan([[2, 2]], [6], [1])["copies"].T.tolist() == [[2, 0, 2]]
    assert plan([[1, 2]], [6], [1], reserved=[0, 0, 1, 0, 0, 0])["copies"].T.tolist() == [[2, 0, 2]]
    # full pages are shared by any number
    assert plan([[1, -1], [1, -1]], [4, 4], [1, 1])["table"].tolist() == [[1, 0], [1, 2]]


def test_the_exclusive_plan_refuses_what_the_other_refuses(ea):
    P = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(12)]     # never dereferenced

    def call(**kw):
        a = dict(table=P[0], table_stride=20, columns=20, lengths=P[1], B_old=5, parents=P[2], counts=P[3], reserved=None, pages=100, page_size=16, B=7, T=3,
                 new_table=P[4], new_lengths=P[5], granted=P[6], slots=P[7], copies=P[8], free_pages=P[9], workspace=P[10], workspace_bytes=1 << 30)
        a.update(kw)
        return ea.el_attn_plan_pages_exclusive(**a)
    for bad in (dict(table=None), dict(copies=None), dict(table=ctypes.c_void_p(0x100002)), dict(slots=ctypes.c_void_p(0x100004)), dict(columns=0), dict(table_stride=19), dict(B=0),
                dict(B_old=0), dict(pages=(1 << 24) + 1), dict(page_size=1 << 28), dict(T=0), dict(parents=None), dict(workspace=ctypes.c_void_p(0x100008))):
        assert call(**bad) == ea.EL_ERR_INVALID_ARG, bad
    need = ea.el_attn_plan_workspace_bytes(7, 100)
    assert call(workspace_bytes=need - 1) == ea.EL_ERR_WORKSPACE and call(workspace=None) == ea.EL_ERR_WORKSPACE
