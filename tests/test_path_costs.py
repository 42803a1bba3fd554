"""Mean cost of shortest paths: a2a_path_costs, the gradient of the link loads' total cost by the demands.

Tolerances, counted before the first run: a level adds a cost, multiplies by a path count, adds up to d products and path counts
(exact below 2^53) and divides, 2 d + 4 roundings of 2^-53; costs are positive or taken by their size, so they add up over the levels."""
from fractions import Fraction

import numpy as np
import pytest

import a2a_inputs as gen
import dispatch_cases as dc
from helpers import tiny_graphs

gpu = pytest.mark.gpu


def tolerance(col, n, depth):
    d = np.bincount(col, minlength=n).max(initial=0)
    return (depth + 1) * (2 * d + 4) * 2.0 ** -53


@pytest.mark.parametrize("name", sorted(tiny_graphs()))
def test_definition_against_path_enumeration(oracle, name):
    """Every shortest path written out, in exact fractions; and the gradient of the loads' cost: loads are linear in the demands."""
    from oracle import brute_force
    rp, col = tiny_graphs()[name]
    N, E = len(rp) - 1, len(col)
    w = [Fraction(3 * a % 7 - 2) for a in range(E)]
    o = oracle.run(rp, col, want_dist=True, want_sigma=True)
    got = dc.path_costs(rp, col, o.dist, o.sigma.astype(np.float64), [float(x) for x in w])
    for s in range(N):
        for t in range(N):
            paths = brute_force.shortest_paths(rp, col, o.dist, s, t) if s != t else []
            want = sum(sum(w[a] for a in p) for p in paths) / Fraction(max(1, len(paths)))
            assert got[s, t] == pytest.approx(float(want), rel=1e-13, abs=1e-13)
    demand = np.zeros((N, N))
    base, _ = oracle.run_demand(rp, col, demand)
    for s, t in ((0, N - 1), (1, 0)):
        demand[s, t] = 5.0
        more, _ = oracle.run_demand(rp, col, demand)
        assert (np.array([float(x) for x in w]) * (more - base)).sum() == pytest.approx(5.0 * got[s, t], rel=1e-12, abs=1e-12)
        demand[s, t] = 0.0


@pytest.fixture(scope="module")
def a2a():
    import torch
    assert torch.cuda.is_available()
    import paper_2309_13541_amd as lib
    lib.load_library()
    return lib


def costs_of(a2a, topo, link_cost, s0=0, count=None):
    """dist, sigma and cost of a source range, by the library."""
    import torch
    count = topo.N - s0 if count is None else count
    dist = torch.empty((count, topo.N), dtype=torch.int32, device="cuda")
    sigma = torch.empty((count, topo.N), dtype=torch.float64, device="cuda")
    cost = torch.full((count + 1, topo.N), -7.0, dtype=torch.float64, device="cuda")
    topo.distances(s0, count, dist=dist, sigma=sigma, workspace=topo.alloc_workspace(count, a2a.WS_SIGMA))
    ws = topo.alloc_workspace(count, a2a.WS_COSTS)
    first = None
    for _ in range(2):
        ws.random_(0, 255)
        topo.path_costs(s0, count, dist=dist, sigma=sigma, link_cost=link_cost, cost=cost[:count], workspace=ws)
        assert first is None or torch.equal(first, cost)
        first = cost.clone()
        cost[:count] = 3.0
    assert (first[count] == -7.0).all()
    return dist, sigma, first[:count]


GRAPHS = {
    **tiny_graphs(),
    "torus8x8": gen.torus([8, 8]),
    "hypercube7": gen.hypercube(7),
    "kautz81": gen.imase_itoh(81, 8),
    "random300": gen.random_regular(300, 4, 5),
    "two_parts": gen.csr_from_rows([[1, 2], [2, 0], [0]] + [[4 + (i + 1) % 60, 4 + (i + 7) % 60] for i in range(60)] + [[3]]),
    "hub": gen.csr_from_rows([list(range(1, 80))] + [[0, (i + 1) % 80] for i in range(1, 79)] + [[0]]),
    "ring150": gen.ring(150),
    "ladder": gen.torus([2, 80]),
    "random1500": gen.random_regular(1500, 3, 8),
}


@gpu
@pytest.mark.parametrize("name", sorted(GRAPHS))
def test_against_the_definition(a2a, oracle, name):
    rp, col = GRAPHS[name]
    N, E = len(rp) - 1, len(col)
    rng = np.random.default_rng(N)
    topo = a2a.Topology(rp, col)
    o = oracle.run(rp, col, want_dist=True, want_sigma=True)
    sigma = o.sigma.astype(np.float64)
    import torch
    for w in (rng.random(E) + 0.1, rng.normal(size=E), None):
        _, _, got = costs_of(a2a, topo, None if w is None else torch.from_numpy(w).cuda())
        ones = np.ones(E) if w is None else w
        want = dc.path_costs(rp, col, o.dist, sigma, ones)
        size = dc.path_costs(rp, col, o.dist, sigma, np.abs(ones))
        tol = tolerance(col, N, int(o.dist.max(initial=0)))
        assert (np.abs(got.cpu().numpy() - want) <= 2 * tol * size).all()
    assert np.abs(got.cpu().numpy() - np.maximum(o.dist, 0)).max() <= tol * o.dist.max()  # cost 1 a link: hop distances
    topo.close()


def by_levels(rp, col, dist, sigma, w):
    """The definition on the device, a level of all sources at a time."""
    import torch
    start = torch.from_numpy(np.repeat(np.arange(len(rp) - 1), np.diff(rp))).cuda()
    end = torch.from_numpy(col.astype(np.int64)).cuda()
    total = torch.zeros_like(sigma)
    for level in range(int(dist.max())):
        on = (dist[:, start] == level) & (dist[:, end] == level + 1)
        total.index_add_(1, end, torch.where(on, total[:, start] + sigma[:, start] * w, 0.0))
    return total / sigma.clamp(min=1.0)


@gpu
@pytest.mark.parametrize("shape", [("random", 4500, 9, 100, 700), ("random", 8192, 4, 0, 300), ("random", 9000, 3, 8800, 200),
                                   ("random", 17000, 4, 16900, 100), ("random", 20011, 5, 7, 65), ("random", 65536, 8, 65500, 36),
                                   ("random", 65537, 3, 0, 20), ("random", 70001, 2, 70000, 1), ("random", 600, 17, 0, 600),
                                   ("random", 9001, 20, 500, 40), ("torus", (13, 17, 19), 0, 1000, 300), ("torus", (90, 90), 0, 0, 70),
                                   ("torus", (2, 5000), 0, 77, 9), ("torus", (40, 41, 42), 0, 500, 20),
                                   ("random", 9000, 10, 0, 100), ("random", 9000, 16, 8900, 64), ("random", 17000, 10, 0, 70),
                                   ("random", 17000, 12, 5, 80), ("random", 16385, 6, 16000, 385), ("random", 40000, 3, 39000, 700),
                                   ("torus", (128, 128), 0, 0, 40), ("torus", (8, 8, 8, 8), 0, 0, 4096),
                                   ("kautz", 12000, 4, 100, 600), ("kautz", 10000, 5, 0, 512), ("kautz", 10000, 7, 9400, 600),
                                   ("kautz", 8500, 10, 0, 530), ("kautz", 9000, 11, 8000, 700), ("kautz", 16384, 4, 0, 16384),
                                   ("random", 9000, 4, 0, 600), ("random", 12000, 16, 0, 512)], ids=str)
def test_larger(a2a, shape):
    """Of every size of a topology's state, a range of sources; against the definition on the device."""
    import torch
    kind, size, d, s0, count = shape
    rp, col = gen.torus(size) if kind == "torus" else (gen.random_regular if kind == "random" else gen.imase_itoh)(size, d, *[5] * (kind == "random"))
    print(f"case {shape}", flush=True)
    topo = a2a.Topology(rp, col)
    w = torch.rand(topo.E, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) + 0.01
    dist, sigma, cost = costs_of(a2a, topo, w, s0, count)
    want = by_levels(rp, col, dist, sigma, w)
    assert ((cost - want).abs() <= 2 * tolerance(col, topo.N, int(dist.max())) * want).all()
    assert float(cost.max()) > 0
    topo.close()


@gpu
@pytest.mark.parametrize("make", [lambda: gen.torus([6, 7, 8]), lambda: gen.imase_itoh(2000, 4), lambda: gen.random_regular(9000, 6, 2)])
def test_gradient_of_the_loads_cost(a2a, make):
    """sum_a w_a load_a = sum_{s,t} demand(s,t) cost(s,t), with the loads of a2a_link_loads_demand; and differences: one pair more."""
    import torch
    rp, col = make()
    topo = a2a.Topology(rp, col)
    g = torch.Generator("cuda").manual_seed(3)
    count = min(topo.N, 500)
    demand = torch.rand((topo.N, count), dtype=torch.float64, device="cuda", generator=g)
    w = torch.rand(topo.E, dtype=torch.float64, device="cuda", generator=g)
    _, _, cost = costs_of(a2a, topo, w, 0, count)
    load = torch.empty(topo.E, dtype=torch.float64, device="cuda")
    ws = topo.alloc_workspace(count, a2a.WS_LOADS)

    def total():
        topo.link_loads_demand(0, count, demand=demand, load=load, workspace=ws)
        return float((w * load).sum())

    at = total()
    assert at == pytest.approx(float((demand.t() * cost).sum()), rel=1e-9)  # the loads' own bound
    for s, t in ((0, topo.N - 1), (count - 1, 5), (7, 7)):
        demand[t, s] += at
        assert total() - at == pytest.approx(at * float(cost[s, t]), rel=1e-8, abs=1e-8 * at)
        demand[t, s] -= at
    topo.close()


@gpu
def test_other_distances_stay_in_bounds(a2a):
    """Distances and counts of another topology, and numbers that are none: some costs, no access out of bounds."""
    import torch
    for n, d, count in ((700, 4, 5), (4000, 4, 5), (8000, 3, 5), (9000, 3, 5), (9000, 3, 520), (20011, 3, 5), (20011, 3, 70), (66000, 2, 5)):
        topo = a2a.Topology(*gen.random_regular(n, d, 1))
        g = torch.Generator("cuda").manual_seed(2)
        dist = torch.randint(-2**31, 2**31 - 1, (count, n), dtype=torch.int32, device="cuda", generator=g)
        dist[1:3] = torch.randint(-3, topo.level_bound + 3, (2, n), dtype=torch.int32, device="cuda", generator=g)
        sigma = torch.randn((count, n), dtype=torch.float64, device="cuda", generator=g)
        cost = torch.full((count + 2, n), -7.0, dtype=torch.float64, device="cuda")
        topo.path_costs(0, count, dist=dist, sigma=sigma, cost=cost[1:-1], workspace=topo.alloc_workspace(count, a2a.WS_COSTS))
        assert (cost[0] == -7.0).all() and (cost[-1] == -7.0).all()
        topo.close()


@gpu
def test_no_links_no_sources_refusals(a2a):
    import torch
    topo = a2a.Topology(np.zeros(4, np.int32), np.zeros(0, np.int32))
    dist, _, cost = costs_of(a2a, topo, None)
    assert not cost.any() and (dist < 0).sum() == 6
    topo.close()
    topo = a2a.Topology(*gen.torus([3, 3]))
    dist, sigma, cost = costs_of(a2a, topo, None)
    ws = topo.alloc_workspace(9, a2a.WS_COSTS)
    good = dict(dist=dist, sigma=sigma, cost=torch.full_like(cost, -7.0), workspace=ws)
    topo.path_costs(3, 0, dist=dist[:0], sigma=sigma[:0], cost=cost[:0], workspace=None)
    for other in (dict(dist=dist.long()), dict(sigma=sigma.float()), dict(cost=cost[:8]), dict(dist=dist.t()), dict(workspace=None),
                  dict(link_cost=torch.ones(35, dtype=torch.float64, device="cuda")), dict(link_cost=torch.ones(36, device="cuda"))):
        with pytest.raises(a2a.A2AError):
            topo.path_costs(0, 9, **{**good, **other})
    for s0, n in ((1, 9), (-1, 9)):
        with pytest.raises(a2a.A2AError):
            topo.path_costs(s0, n, **good)
    with pytest.raises(a2a.A2AError) as e:
        topo.path_costs(0, 9, **{**good, "workspace": ws[:0]})
    torch.cuda.synchronize()
    assert (good["cost"] == -7.0).all()
    topo.close()


@gpu
def test_the_whole_way(a2a, oracle):
    """A router's choices to the schedule's time and back: demands of the dispatch, link loads, prices of the loaded links,
    costs of the pairs, the balance loss weighted by them and its gradient; on a stream of its own, then recorded and replayed."""
    import torch
    rp, col = gen.torus([4, 6])
    N, T, k, X = 24, 2000, 3, 48
    topo = a2a.Topology(rp, col)
    rng = np.random.default_rng(12)
    begin = dc.begins("ragged", N, T, rng)
    place = rng.integers(0, N, X).astype(np.int32)
    z = rng.normal(size=(T, X)).astype(np.float32)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        f = dict(device="cuda")
        d_z, d_begin, d_place = torch.from_numpy(z).cuda(), torch.from_numpy(begin).cuda(), torch.from_numpy(place).cuda()
        c = d_z.topk(k, dim=1).indices
        dist = torch.empty((N, N), dtype=torch.int32, **f)
        sigma, cost, demand = (torch.empty((N, N), dtype=torch.float64, **f) for _ in range(3))
        load = torch.empty(topo.E, dtype=torch.float64, **f)
        loss, grad = torch.empty(1, **f), torch.empty_like(d_z)
        counts, sums = torch.empty((N, X), dtype=torch.int32, **f), torch.empty((N, X), **f)
        rows = torch.empty(N, dtype=torch.int32, **f)
        ws = topo.alloc_workspace(N, a2a.WS_LOADS), topo.alloc_workspace(N, a2a.WS_SIGMA), topo.alloc_workspace(N, a2a.WS_COSTS)
        ws_b = topo.alloc_balance_workspace(N, tokens=T, experts=X)

        def call(stream=None):
            topo.dispatch_demand(N, choices=c, host_begin=d_begin, experts=X, expert_host=d_place, demand=demand, stream=stream)
            topo.link_loads_demand(0, N, demand=demand, load=load, workspace=ws[0], stream=stream)
            topo.distances(0, N, dist=dist, sigma=sigma, workspace=ws[1], stream=stream)
            topo.path_costs(0, N, dist=dist, sigma=sigma, link_cost=load, cost=cost, workspace=ws[2], stream=stream)
            w = dict(cost=cost, expert_host=d_place, stream=stream)
            topo.balance_loss(N, logits=d_z, choices=c, host_begin=d_begin, loss=loss, counts=counts, prob_sums=sums, rows=rows,
                              workspace=ws_b, **w)
            topo.balance_loss_grad(N, logits=d_z, choices_per_token=k, host_begin=d_begin, counts=counts, rows=rows, grad=grad, **w)

        call(st)
    st.synchronize()
    outs = [demand, load, cost, loss, counts, sums, rows, grad]
    eager = [x.clone() for x in outs]
    ids = c.cpu().numpy()
    want_demand = dc.demand(begin, ids, X, place, N, False)
    assert np.array_equal(demand.cpu().numpy(), want_demand)
    want_load, _ = oracle.run_demand(rp, col, np.ascontiguousarray(want_demand.T))
    np.testing.assert_allclose(load.cpu().numpy(), want_load, rtol=1e-9)
    o = oracle.run(rp, col, want_dist=True, want_sigma=True)
    want_cost = dc.path_costs(rp, col, o.dist, o.sigma.astype(np.float64), want_load)
    np.testing.assert_allclose(cost.cpu().numpy(), want_cost, rtol=3e-9)
    r = dc.balance(z.astype(np.float64), begin, ids, dc.weights(want_cost, place, N, X))
    assert float(loss) == pytest.approx(r["loss"], rel=3e-5)
    want = dc.balance_grad(r)
    assert np.linalg.norm(grad.cpu().numpy() - want) <= 3e-5 * np.linalg.norm(want)
    # what the loss is: the links' price of the traffic that the probabilities ask for, by the choices made
    assert float((load * load).sum()) == pytest.approx(float((demand.t() * cost).sum()), rel=1e-9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(4):
        for x in outs:
            x.fill_(2)
        for x in (*ws, ws_b):
            x.random_(0, 255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), rep
    del graph
    topo.close()
