"""Counts and demands of a router's choices: a2a_dispatch_counts, a2a_dispatch_demand.  Whole numbers: equal."""
import numpy as np
import pytest

import a2a_inputs as gen
import dispatch_cases as dc

gpu = pytest.mark.gpu


def device(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


@pytest.fixture(scope="module")
def a2a():
    import torch
    assert torch.cuda.is_available()
    import paper_2309_13541_amd as lib
    lib.load_library()
    return lib


def ring(a2a, n):
    return a2a.Topology(*gen.ring(n)) if n > 1 else a2a.Topology(np.zeros(2, np.int32), np.zeros(0, np.int32))


def test_the_cases_themselves():
    """One case by hand."""
    begin = np.array([1, 3, 3, 5])
    c = np.array([[0, 1], [1, 1], [2, -1], [3, 9], [0, 2], [0, 0]])
    assert dc.sources_of(begin, 6).tolist() == [-1, 0, 0, 2, 2, -1]
    assert dc.counts(begin, c, 4).tolist() == [[0, 2, 1, 0], [0] * 4, [1, 0, 1, 1]]
    place = np.array([2, 0, 2, -1])
    assert dc.demand(begin, c, 4, place, 3, False).tolist() == [[2, 0, 0], [0, 0, 0], [1, 0, 2]]
    assert dc.demand(begin, c, 4, place, 3, True).tolist() == [[1, 0, 0], [0, 0, 0], [1, 0, 1]]


SHAPES = [  # sources, tokens, k, experts
    (1, 1, 1, 1), (1, 0, 3, 5), (7, 1, 2, 9), (64, 96, 2, 64), (5, 1000, 6, 7), (1, 5000, 8, 300), (300, 77, 3, 1025),
    (33, 4099, 4, 257), (700, 2000, 1, 40), (3, 300, 64, 5000), (1100, 2300, 5, 130),
]


@gpu
@pytest.mark.parametrize("kind", ["even", "ragged", "one", "gaps", "past"])
@pytest.mark.parametrize("dtype", [np.int32, np.int64])
@pytest.mark.parametrize("shape", SHAPES)
def test_counts(a2a, shape, dtype, kind):
    import torch
    S, T, k, X = shape
    rng = np.random.default_rng(S + T)
    begin, c = dc.begins(kind, S, T, rng), dc.choices(rng, T, k, X, dtype)
    topo = ring(a2a, 3)
    got = torch.full((S + 1, X), -7, dtype=torch.int32, device="cuda")
    for _ in range(2):
        topo.dispatch_counts(S, choices=device(c), host_begin=device(begin), experts=X, counts=got[:S])
        assert np.array_equal(got[:S].cpu().numpy(), dc.counts(begin, c, X))
        got[:S] = 99
    assert (got[S] == -7).all()
    topo.close()


@gpu
@pytest.mark.parametrize("once", [False, True])
@pytest.mark.parametrize("kind", ["even", "ragged", "one", "past"])
@pytest.mark.parametrize("shape", [
    (64, 64, 96, 2, 64), (1, 1, 9, 2, 3), (81, 81, 3000, 6, 405), (81, 17, 500, 4, 81), (300, 300, 2000, 8, 100),
    (1000, 1, 3000, 3, 2000), (1030, 9, 4000, 4, 1030), (600, 600, 1, 1, 600), (40, 40, 0, 2, 10), (9000, 20, 700, 5, 9000),
    (40, 40, 600, 20, 90), (20, 3, 5000, 64, 33), (600, 600, 900, 9, 30), (2100, 2100, 6000, 3, 2100)])
def test_demand(a2a, shape, kind, once):
    import torch
    N, S, T, k, X = shape
    rng = np.random.default_rng(N + T)
    topo = ring(a2a, N)
    place = rng.integers(-2, N + 3, X).astype(np.int32) if X != N else None
    for dtype in (np.int32, np.int64):
        begin, c = dc.begins(kind, S, T, rng), dc.choices(rng, T, k, X, dtype)
        got = torch.full((N + 1, S), -7.0, dtype=torch.float64, device="cuda")
        topo.dispatch_demand(S, choices=device(c), host_begin=device(begin), experts=X, once=once, demand=got[:N],
                             expert_host=None if place is None else device(place))
        want = dc.demand(begin, c, X, place, N, once)
        assert np.array_equal(got[:N].cpu().numpy(), want)
        assert (got[N] == -7.0).all()
    topo.close()


@gpu
def test_rows_of_choices_apart(a2a):
    """Choices as columns of a wider matrix, not at its first: rows that are no multiple of 8 bytes apart."""
    import torch
    rng = np.random.default_rng(3)
    N, T, k, X = 50, 700, 3, 80
    begin = dc.begins("ragged", N, T, rng)
    place = rng.integers(0, N, X).astype(np.int32)
    topo = ring(a2a, N)
    for dtype in (np.int32, np.int64):
        wide = device(dc.choices(rng, T, 11, X, dtype))
        view = wide[:, 5:5 + k]
        c = view.cpu().numpy()
        counts = torch.empty((N, X), dtype=torch.int32, device="cuda")
        demand = torch.empty((N, N), dtype=torch.float64, device="cuda")
        topo.dispatch_counts(N, choices=view, host_begin=device(begin), experts=X, counts=counts)
        topo.dispatch_demand(N, choices=view, host_begin=device(begin), experts=X, expert_host=device(place), once=True, demand=demand)
        assert np.array_equal(counts.cpu().numpy(), dc.counts(begin, c, X))
        assert np.array_equal(demand.cpu().numpy(), dc.demand(begin, c, X, place, N, True))
    topo.close()


@gpu
def test_many_tokens_of_one_pair(a2a):
    """All choices on one expert: every addition meets the same place."""
    import torch
    T, k = 200003, 8
    topo = ring(a2a, 4)
    c = torch.full((T, k), 2, dtype=torch.int32, device="cuda")
    begin = torch.tensor([0, 0, T - 1, T, T], device="cuda")
    counts = torch.empty((4, 5), dtype=torch.int32, device="cuda")
    demand = torch.empty((4, 4), dtype=torch.float64, device="cuda")
    topo.dispatch_counts(4, choices=c, host_begin=begin, experts=5, counts=counts)
    want = torch.zeros((4, 5), dtype=torch.int32)
    want[1, 2], want[2, 2] = (T - 1) * k, k
    assert torch.equal(counts.cpu(), want)
    for once in (False, True):
        topo.dispatch_demand(4, choices=c, host_begin=begin, experts=5, once=once, demand=demand)
        want = torch.zeros((4, 4), dtype=torch.float64)
        want[2, 1], want[2, 2] = (T - 1) * (1 if once else k), 1 if once else k
        assert torch.equal(demand.cpu(), want)
    topo.close()


@gpu
def test_many_choices_of_a_band(a2a):
    """More than 65535 choices of sources that one workgroup has: cells of 32 bits, and the rows in two halves."""
    import torch
    N, T, k = 600, 30000, 4
    topo = ring(a2a, N)
    g = torch.Generator("cuda").manual_seed(5)
    c = torch.randint(-1, N, (T, k), device="cuda", generator=g)
    begin = torch.zeros(N + 1, dtype=torch.int64, device="cuda")
    begin[300:] = T - 500  # source 299 has nearly all
    begin[400:] = T
    source = torch.searchsorted(begin, torch.arange(T, device="cuda"), right=True) - 1
    demand = torch.full((N, N), -7.0, dtype=torch.float64, device="cuda")
    counts = torch.full((N, N), -7, dtype=torch.int32, device="cuda")
    topo.dispatch_demand(N, choices=c, host_begin=begin, experts=N, demand=demand)
    topo.dispatch_counts(N, choices=c, host_begin=begin, experts=N, counts=counts)
    want = torch.bincount((source[:, None] * N + c)[c >= 0], minlength=N * N).view(N, N)
    assert torch.equal(counts.long(), want) and torch.equal(demand, want.t().double())
    topo.close()


@gpu
def test_decreasing_begins_stay_in_bounds(a2a):
    """host_begin that is none: some numbers, no access out of bounds."""
    import torch
    g = torch.Generator("cuda").manual_seed(6)
    S, T, k, X = 300, 2000, 2, 40
    topo = ring(a2a, S)
    c = torch.randint(0, X, (T, k), device="cuda", generator=g)
    z = torch.randn((T, X), device="cuda", generator=g)
    for sources in (S, 4):
        begin = torch.randint(-T, 3 * T, (sources + 1,), device="cuda", generator=g)
        counts = torch.full((sources + 2, X), -7, dtype=torch.int32, device="cuda")
        demand = torch.full((S + 2, sources), -7.0, dtype=torch.float64, device="cuda")
        topo.dispatch_counts(sources, choices=c, host_begin=begin, experts=X, counts=counts[1:-1])
        topo.dispatch_demand(sources, choices=c, host_begin=begin, experts=X, once=True, demand=demand[1:-1])
        loss, sums = torch.empty(1, device="cuda"), torch.full((sources + 2, X), -7.0, device="cuda")
        rows = torch.full((sources + 2,), -7, dtype=torch.int32, device="cuda")
        ws = topo.alloc_balance_workspace(sources, tokens=T, experts=X).zero_()
        grad = torch.full((T + 2, X), -7.0, device="cuda")
        topo.balance_loss(sources, logits=z, choices=c, host_begin=begin, loss=loss, counts=counts[1:-1], prob_sums=sums[1:-1],
                          rows=rows[1:-1], workspace=ws)
        topo.balance_loss_grad(sources, logits=z, choices_per_token=k, host_begin=begin, counts=counts[1:-1], rows=rows[1:-1],
                               grad=grad[1:-1])
        for x in (counts, demand, sums, rows, grad):
            assert (x[0] == -7).all() and (x[-1] == -7).all()
    topo.close()


@gpu
def test_two_streams_at_once(a2a):
    """Counts, demands, loss and gradient of two batches on two streams of one handle, each with its own buffers: what each gives alone."""
    import torch
    S, T, k, X = 64, 6000, 4, 96
    topo = ring(a2a, S)
    streams = [torch.cuda.Stream() for _ in range(2)]

    def batch(seed):
        g = torch.Generator("cuda").manual_seed(seed)
        z = torch.randn((T, X), device="cuda", generator=g)
        return dict(z=z, c=z.topk(k, dim=1).indices, begin=torch.linspace(0, T, S + 1, device="cuda").long(),
                    place=torch.randint(0, S, (X,), device="cuda", generator=g, dtype=torch.int32),
                    ws=topo.alloc_balance_workspace(S, tokens=T, experts=X))

    def call(b, stream=None):
        f = dict(device="cuda")
        demand, loss = torch.empty((S, S), dtype=torch.float64, **f), torch.empty(1, **f)
        counts, sums = torch.empty((S, X), dtype=torch.int32, **f), torch.empty((S, X), **f)
        rows, grad = torch.empty(S, dtype=torch.int32, **f), torch.empty_like(b["z"])
        topo.dispatch_demand(S, choices=b["c"], host_begin=b["begin"], experts=X, expert_host=b["place"], demand=demand, stream=stream)
        w = dict(cost=demand.t().contiguous(), expert_host=b["place"], stream=stream)
        topo.balance_loss(S, logits=b["z"], choices=b["c"], host_begin=b["begin"], loss=loss, counts=counts, prob_sums=sums, rows=rows,
                          workspace=b["ws"], **w)
        topo.balance_loss_grad(S, logits=b["z"], choices_per_token=k, host_begin=b["begin"], counts=counts, rows=rows, grad=grad, **w)
        return [demand, loss, counts, sums, rows, grad, w["cost"]]

    batches = [batch(1), batch(2)]
    torch.cuda.synchronize()
    want = [call(b) for b in batches]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for b, st in zip(batches, streams):
            with torch.cuda.stream(st):
                got.append(call(b, st))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))
    topo.close()


@gpu
def test_refusals(a2a):
    """Before anything is enqueued: the outputs stay as they are."""
    import torch
    topo = ring(a2a, 6)
    S, T, k, X = 6, 10, 2, 8

    def tensors():
        return dict(choices=torch.zeros((T, k), dtype=torch.int64, device="cuda"),
                    host_begin=torch.zeros(S + 1, dtype=torch.int64, device="cuda"), experts=X,
                    counts=torch.full((S, X), -7, dtype=torch.int32, device="cuda"))

    def refused(**other):
        a = {**tensors(), **other}
        with pytest.raises(a2a.A2AError):
            topo.dispatch_counts(S, **a)
        torch.cuda.synchronize()
        assert (a["counts"] == -7).all()

    refused(choices=torch.zeros((T, k), dtype=torch.int16, device="cuda"))
    refused(choices=torch.zeros((k, T), dtype=torch.int64, device="cuda").t())
    refused(choices=torch.zeros((T, k), dtype=torch.int64))
    refused(choices=torch.zeros((T, 65), dtype=torch.int64, device="cuda"))
    refused(choices=torch.zeros((1, k), dtype=torch.int64, device="cuda").expand(T, k))
    refused(host_begin=torch.zeros(S, dtype=torch.int64, device="cuda"))
    refused(host_begin=torch.zeros(S + 1, dtype=torch.int32, device="cuda"))
    refused(experts=X + 1)
    refused(counts=torch.full((S, 2 * X), -7, dtype=torch.int32, device="cuda")[:, ::2])
    with pytest.raises(a2a.A2AError):  # more sources than hosts
        topo.dispatch_demand(7, choices=tensors()["choices"], host_begin=torch.zeros(8, dtype=torch.int64, device="cuda"), experts=X,
                             demand=torch.zeros((6, 7), dtype=torch.float64, device="cuda"))
    topo.close()


@gpu
def test_replayed(a2a):
    """Recorded into a graph and replayed on other choices each time."""
    import torch
    rng = np.random.default_rng(8)
    N, T, k, X = 90, 900, 4, 120
    topo = ring(a2a, N)
    c = device(dc.choices(rng, T, k, X, np.int64))
    begin = device(dc.begins("ragged", N, T, rng))
    place = device(rng.integers(0, N, X).astype(np.int32))
    counts = torch.empty((N, X), dtype=torch.int32, device="cuda")
    demand = torch.empty((N, N), dtype=torch.float64, device="cuda")

    def call():
        topo.dispatch_counts(N, choices=c, host_begin=begin, experts=X, counts=counts)
        topo.dispatch_demand(N, choices=c, host_begin=begin, experts=X, expert_host=place, demand=demand)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(4):
        new = dc.choices(rng, T, k, X, np.int64)
        c.copy_(torch.from_numpy(new))
        counts.fill_(-1)
        demand.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b, p = begin.cpu().numpy(), place.cpu().numpy()
        assert np.array_equal(counts.cpu().numpy(), dc.counts(b, new, X)), rep
        assert np.array_equal(demand.cpu().numpy(), dc.demand(b, new, X, p, N, False)), rep
    del graph
    topo.close()
