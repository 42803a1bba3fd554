"""Gradient of rows that are no token (all -infinity): 0, whatever the other factors of the gradient are."""
import pytest

import a2a_inputs as gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("factor", ["upstream inf", "upstream nan", "cost inf", "cost nan", "coefficient past a float"])
@pytest.mark.parametrize("type_", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("experts", [8, 24, 31, 160, 500, 2048])
def test_no_token_has_no_gradient(experts, type_, factor):
    """A step whose loss has overflowed (an infinite gradient from above), a price that is none: padded rows stay 0, the others are
    the formula's."""
    import torch
    import paper_2309_13541_amd as a2a
    f = dict(device="cuda")
    topo = a2a.Topology(*gen.ring(5))
    S, T, k, X = 5, 300, 2, experts
    z = torch.randn((T, X), generator=torch.Generator("cuda").manual_seed(X), **f).to(getattr(torch, type_))
    empty = torch.arange(T, **f) % 3 == 1
    z[empty] = -torch.inf
    c = torch.arange(2 * T, **f).view(T, k) % X
    begin = torch.tensor([0, 50, 130, 200, 290, T], **f)
    up = torch.full((1,), {"upstream inf": torch.inf, "upstream nan": torch.nan, "coefficient past a float": 1e38}.get(factor, 1.0), **f)
    cost = torch.ones((S, 5), dtype=torch.float64, **f)
    if factor == "coefficient past a float":
        cost[:] = 1e9
    elif factor.startswith("cost"):
        cost[1, 2] = torch.inf if factor == "cost inf" else torch.nan
    place = torch.arange(X, **f).int() % 5
    loss, counts = torch.empty(1, **f), torch.empty((S, X), dtype=torch.int32, **f)
    sums, rows = torch.empty((S, X), **f), torch.empty(S, dtype=torch.int32, **f)
    ws = topo.alloc_balance_workspace(S, tokens=T, experts=X)
    grad = torch.full_like(z, -7.0)
    w = dict(cost=cost, expert_host=place)
    topo.balance_loss(S, logits=z, choices=c, host_begin=begin, loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws, **w)
    topo.balance_loss_grad(S, logits=z, choices_per_token=k, host_begin=begin, counts=counts, rows=rows, upstream=up, grad=grad, **w)
    assert not grad[empty].any()
    source = torch.searchsorted(begin, torch.arange(T, **f), right=True) - 1
    other = source == 1 if factor.startswith("cost") else torch.ones_like(empty)
    assert not torch.isfinite(grad[other & ~empty]).all(1).any()  # inf * p, less its mean: no number
    assert torch.isfinite(grad[~other]).all()
    assert rows.tolist() == torch.bincount(source[~empty], minlength=S).tolist()
    topo.close()
