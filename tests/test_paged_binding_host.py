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
