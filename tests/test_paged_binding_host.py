"""The binding of the paged cache without a GPU."""
import pytest
import torch
import torch.autograd.forward_ad as fw

from paper_2105_04779_amd import el_attn


def test_a_cache_keeps_the_pools_that_it_was_made_of():
    """The kernels are given the addresses that the constructor saw: another tensor in their place would be ignored."""
    cache = object.__new__(el_attn.PagedCache)
    for name in ("K", "V"):
        with pytest.raises(AttributeError):
            setattr(cache, name, torch.zeros((4, 16, 2, 64)))


def test_what_asks_for_a_derivative_is_refused():
    x, cpu = torch.zeros(3), torch.device("cpu")
    el_attn._check_values("x", x, cpu, torch.float32)
    with pytest.raises(ValueError, match="gradient"):
        el_attn._check_values("x", x.clone().requires_grad_(), cpu, torch.float32)
    with torch.no_grad():
        el_attn._check_values("x", x.clone().requires_grad_(), cpu, torch.float32)
    with fw.dual_level():
        dual = fw.make_dual(x, torch.ones(3))
        with pytest.raises(ValueError, match="tangent"):
            el_attn._check_values("x", dual, cpu, torch.float32)
        with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
            el_attn._check_values("x", dual, cpu, torch.float32)
        el_attn._check_values("x", x, cpu, torch.float32)


def test_strides_whose_places_pass_the_address_space_are_refused():
    """Each stride is one that a call takes, and the last row lies beyond 2^48 bytes: an address formed of it would have wrapped."""
    import ctypes
    ea, I = el_attn, el_attn.EL_ERR_INVALID_ARG
    P = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(8)]      # never dereferenced
    c = ea.ElAttnPages(P[0], P[1], 16 * 128, 128, 128, 40, 16, 1, 128, ea.EL_BF16)
    attend = dict(table=P[2], table_stride=10, table_pages=10, lengths=P[3], queries=ctypes.c_void_p(1 << 45), query_stride=128, heads=1,
                  rule=ea.ElAttnScoreRule(0.1, 0.0, 0, None), out=ctypes.c_void_p(1 << 40), out_dtype=ea.EL_BF16, lse=None, B=1 << 20, beam=1, n=160,
                  workspace=None, workspace_bytes=0)
    append = dict(table=P[2], table_stride=10, table_pages=10, lengths=P[3], counts=None, K_new=P[4], V_new=P[5], batch_stride=3 * 128,
                  token_stride=128, B=4, T=3)
    scores = dict(dtype=ea.EL_BF16, logits=P[0], row_stride=1000, rows=1 << 20, vocab=999, tokens=P[1], logprob=P[2], entropy=P[3], k=0,
                  top_logprob=None, top_index=None, workspace=None, workspace_bytes=0)
    for bad in (dict(query_stride=1 << 44), dict(query_stride=1 << 40), dict(table_stride=1 << 40), dict(table_stride=1 << 30)):
        assert ea.el_attn_paged_attend(c, **{**attend, **bad}) == I, bad
    for bad in (dict(batch_stride=1 << 44, B=65535), dict(token_stride=1 << 44, T=1 << 23), dict(token_stride=1 << 30, T=1 << 20), dict(table_stride=1 << 40, B=65535)):
        assert ea.el_attn_paged_append(c, **{**append, **bad}) == I, bad
    for bad in (dict(row_stride=1 << 44), dict(row_stride=1 << 40)):
        assert ea.el_attn_score_tokens(**{**scores, **bad}) == I, bad
