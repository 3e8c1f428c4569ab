"""The binding of the paged cache without a GPU."""
import pytest
import torch
import torch.autograd.forward_ad as fw

from paper_2105_04779_amd import el_attn


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
