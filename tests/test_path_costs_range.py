"""a2a_path_costs for more pairs than 32 bits count, by each of the ways that take so many nodes."""
import pytest

import a2a_inputs as gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("make", [lambda: gen.random_regular(65536, 8, 3), lambda: gen.torus([16, 16, 16, 16]), lambda: gen.random_regular(65543, 4, 3)],
                         ids=["random 65536 x 8", "torus 16x16x16x16", "random 65543 x 4"])
def test_pairs_past_32_bits(make):
    import torch
    import paper_2309_13541_amd as a2a
    rp, col = make()
    topo = a2a.Topology(rp, col)
    N, count, part = topo.N, 33000, 1000
    assert N * count > 2**31
    f = dict(device="cuda")
    dist, sigma = torch.empty((count, N), dtype=torch.int32, **f), torch.empty((count, N), dtype=torch.float64, **f)
    ws = topo.alloc_workspace(part, a2a.WS_SIGMA)
    for s in range(0, count, part):
        topo.distances(s, part, dist=dist[s:s + part], sigma=sigma[s:s + part], workspace=ws)
    print("distances there", flush=True)
    ws = topo.alloc_workspace(count, a2a.WS_COSTS)
    cost = torch.full((count, N), -7.0, dtype=torch.float64, **f)
    # (levels + 1) (2 in-links + 4) roundings, as the operator's other tests count them, 32 levels or 16 in-links at the most
    tol = 33 * 36 * 2.0 ** -53
    topo.path_costs(0, count, dist=dist, sigma=sigma, cost=cost, workspace=ws)  # cost 1 a link: hop distances
    for s in range(0, count, part):
        want = dist[s:s + part].clamp(min=0).double()
        assert ((cost[s:s + part] - want).abs() <= tol * want).all(), s
    w = torch.rand(topo.E, dtype=torch.float64, generator=torch.Generator("cuda").manual_seed(1), **f) + 0.01
    topo.path_costs(0, count, dist=dist, sigma=sigma, link_cost=w, cost=cost, workspace=ws)
    for s in (0, 2**31 // N - 1, count - 3):  # rows before and behind the border, and the last
        few = torch.empty((3, N), dtype=torch.float64, **f)
        topo.path_costs(s, 3, dist=dist[s:s + 3].clone(), sigma=sigma[s:s + 3].clone(), link_cost=w, cost=few, workspace=ws)
        assert ((cost[s:s + 3] - few).abs() <= 2 * tol * few).all(), s
        assert float(few.max()) > 1
    topo.close()
