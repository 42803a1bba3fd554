"""a2a_workspace_bytes for several calls at once: flags together, a workspace that holds each of the calls."""
import pytest

import a2a_inputs as gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("make", [lambda: gen.torus([4, 6]), lambda: gen.imase_itoh(3000, 4), lambda: gen.imase_itoh(20000, 5),
                                  lambda: gen.random_regular(600, 17, 2)])
@pytest.mark.parametrize("smallest", [False, True])
def test_one_workspace_for_several_calls(make, smallest):
    import torch
    import paper_2309_13541_amd as a2a
    topo = a2a.Topology(*make())
    n = min(topo.N, 300)
    less = a2a.WS_MINIMAL if smallest else 0
    both = topo.workspace_bytes(n, a2a.WS_COSTS | a2a.WS_LOADS | a2a.WS_SIGMA | less)
    alone = [topo.workspace_bytes(n, x | less) for x in (a2a.WS_COSTS, a2a.WS_LOADS, a2a.WS_SIGMA)]
    assert both == max(both, *alone) and both >= topo.workspace_bytes(n, a2a.WS_LOADS | a2a.WS_SIGMA | less)
    assert topo.workspace_bytes(n, a2a.WS_COSTS | a2a.WS_SSSP | less) >= topo.workspace_bytes(n, a2a.WS_SSSP | less)
    f = dict(device="cuda")
    ws = torch.empty(both, dtype=torch.uint8, **f)
    dist, sigma = torch.empty((n, topo.N), dtype=torch.int32, **f), torch.empty((n, topo.N), dtype=torch.float64, **f)
    cost, load = torch.empty((n, topo.N), dtype=torch.float64, **f), torch.empty(topo.E, dtype=torch.float64, **f)
    topo.distances(0, n, dist=dist, sigma=sigma, workspace=ws)
    topo.link_loads(0, n, load=load, workspace=ws)
    topo.path_costs(0, n, dist=dist, sigma=sigma, cost=cost, workspace=ws)
    # cost 1 a link: the loads' sum and the costs' are both the sum of all distances, each within a rounding or so of every term
    total = float(dist.clamp(min=0).sum())
    assert float(load.sum()) == pytest.approx(total, rel=1e-9) and float(cost.sum()) == pytest.approx(total, rel=1e-9)
    topo.close()
