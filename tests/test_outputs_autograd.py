"""What the dispatch functions and a2a_path_costs write counts for torch as written: a program's own autograd graph that has saved such a
tensor does not go on with what is there now, but says so."""
import numpy as np
import pytest

import a2a_inputs as gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def a2a():
    import torch
    assert torch.cuda.is_available()
    import paper_2309_13541_amd as lib
    lib.load_library()
    return lib


def routed(topo, S=4, T=40, k=2, X=24):
    import torch
    f = dict(device="cuda")
    z = torch.randn((T, X), **f)
    return dict(z=z, c=z.topk(k, dim=1).indices, begin=torch.tensor([0, 9, 20, 20, T], **f), S=S, X=X, k=k,
                loss=torch.zeros(1, **f), counts=torch.zeros((S, X), dtype=torch.int32, **f), sums=torch.zeros((S, X), **f),
                rows=torch.zeros(S, dtype=torch.int32, **f), ws=topo.alloc_balance_workspace(S, tokens=T, experts=X))


def loss_of(topo, r):
    topo.balance_loss(r["S"], logits=r["z"], choices=r["c"], host_begin=r["begin"], loss=r["loss"], counts=r["counts"], prob_sums=r["sums"],
                      rows=r["rows"], workspace=r["ws"])


def test_every_output(a2a):
    import torch
    topo = a2a.Topology(*gen.ring(4))
    r = routed(topo)
    grad, demand = torch.zeros_like(r["z"]), torch.zeros((4, 4), dtype=torch.float64, device="cuda")
    dist = torch.zeros((4, 4), dtype=torch.int32, device="cuda")
    sigma, cost = torch.zeros((4, 4), dtype=torch.float64, device="cuda"), torch.zeros((4, 4), dtype=torch.float64, device="cuda")
    topo.distances(0, 4, dist=dist, sigma=sigma, workspace=topo.alloc_workspace(4, a2a.WS_SIGMA))
    calls = [
        (["counts"], lambda: topo.dispatch_counts(4, choices=r["c"], host_begin=r["begin"], experts=24, counts=r["counts"])),
        ([demand], lambda: topo.dispatch_demand(4, choices=r["c"], host_begin=r["begin"], experts=24, demand=demand)),
        (["loss", "counts", "sums", "rows"], lambda: loss_of(topo, r)),
        ([grad], lambda: topo.balance_loss_grad(4, logits=r["z"], choices_per_token=2, host_begin=r["begin"], counts=r["counts"],
                                                rows=r["rows"], grad=grad)),
        ([cost], lambda: topo.path_costs(0, 4, dist=dist, sigma=sigma, cost=cost, workspace=topo.alloc_workspace(4, a2a.WS_COSTS))),
    ]
    inputs = [r["z"], r["c"], r["begin"], dist, sigma]
    for outs, call in calls:
        outs = [r[x] if isinstance(x, str) else x for x in outs]
        before, kept = [x._version for x in outs], [x._version for x in inputs]
        call()
        assert all(x._version > v for x, v in zip(outs, before)), outs
        assert [x._version for x in inputs] == kept
    with torch.inference_mode():  # these have no counter
        r = routed(topo)
        loss_of(topo, r)
        assert float(r["loss"][0]) > 0
    topo.close()


def test_logits_overwritten_by_their_gradient(a2a):
    """Of a graph that needs the logits again: an error, not another gradient."""
    import torch
    topo = a2a.Topology(*gen.ring(4))
    r = routed(topo)
    weight = torch.ones(24, device="cuda", requires_grad=True)
    own = (r["z"] * weight).sum()  # keeps the logits for its backward pass
    loss_of(topo, r)
    topo.balance_loss_grad(4, logits=r["z"], choices_per_token=2, host_begin=r["begin"], counts=r["counts"], rows=r["rows"], grad=r["z"])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        own.backward()
    topo.close()


def test_graph_of_a_leaf_lives_on(a2a):
    """A gradient into a buffer of its own leaves a graph of the same logits as it was; the caller hands it to the leaf."""
    import torch
    topo = a2a.Topology(*gen.ring(4))
    r = routed(topo)
    leaf = r["z"].clone().requires_grad_()
    own = (leaf * leaf).sum()
    r["z"] = leaf.detach()
    loss_of(topo, r)
    grad = torch.empty_like(r["z"])
    topo.balance_loss_grad(4, logits=r["z"], choices_per_token=2, host_begin=r["begin"], counts=r["counts"], rows=r["rows"], grad=grad)
    own.backward()
    assert torch.equal(leaf.grad, 2 * leaf.detach())
    p = torch.softmax(leaf.detach().double(), 1)
    source = torch.searchsorted(r["begin"], torch.arange(40, device="cuda"), right=True) - 1
    c = (24 * r["counts"].double() / (2 * 40 * r["rows"].clamp(min=1)[:, None]))[source]
    want = p * (c - (p * c).sum(1, keepdim=True))
    # some 90 roundings of 2^-24: 24 additions in the sum and as many in the mean, 40 of an exponent of 8 at most, single ones
    np.testing.assert_allclose(grad.cpu().numpy(), want.cpu().numpy(), rtol=0, atol=2e-5 * float(want.abs().max()))
    topo.close()
