"""Balance loss of a router and its gradient: a2a_balance_loss, a2a_balance_loss_grad, against the definition in 64 bits.

Tolerances, counted before the first run.  eps = 2^-23, a rounding is off by eps / 2 at most.  x = exp(z - top) is off by 2^(its
argument's rounding): of the difference and of the product eps / 2 each and 0.22 eps / 2 for the constant log2(e), of |arg| =
(top - z) log2(e) and times ln 2: 1.54 |arg| eps / 2; and the instruction's own eps.  Values below 2^-149 are 0, so ARG = 230 = 1.54 * 149
bounds it for every element.
The row's sum takes up to 64 additions in a lane and 6 between lanes, its inverse and the product 1 each; a column's sum takes as many
additions as a lane has rows, of a piece of `per` tokens at most per / 4, then 9.  All terms are positive: relative errors add up."""
import numpy as np
import pytest

import a2a_inputs as gen
import dispatch_cases as dc

gpu = pytest.mark.gpu
EPS = 2.0 ** -23
ARG = 230


def column_tolerance(tokens):
    per = max(64, -(-tokens // 2048))
    return (ARG + 2 + 64 + 6 + 2 + per / 4 + 9) * EPS / 2


ROW_TOLERANCE = (ARG + 2 + 64 + 6 + 2 + 64 + 6 + 4) * EPS / 2  # of p (c - dot), whose dot is summed like the row


@pytest.fixture(scope="module")
def a2a():
    import torch
    assert torch.cuda.is_available()
    import paper_2309_13541_amd as lib
    lib.load_library()
    return lib


def device(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


# ---------------------------------------------------------------------------------------------------------
# CPU: the definition
# ---------------------------------------------------------------------------------------------------------

def test_a_router_in_balance_has_loss_one():
    X, T, k = 8, 64, 2
    c = np.stack([np.arange(T) % X, (np.arange(T) + 1) % X], axis=1)
    r = dc.balance(np.zeros((T, X)), np.array([0, T]), c, np.ones((1, X)))
    assert r["loss"] == pytest.approx(1.0, rel=1e-14)
    all_on_one = dc.balance(np.zeros((T, X)) + 50 * (np.arange(X) == 3), np.array([0, T]), np.full((T, k), 3), np.ones((1, X)))
    assert all_on_one["loss"] == pytest.approx(X, rel=1e-12)


def test_gradient_against_differences():
    """Central differences of the loss, with the counts as they are."""
    rng = np.random.default_rng(2)
    S, T, k, X = 3, 17, 2, 6
    z = rng.normal(size=(T, X))
    z[4] = -np.inf
    z[:, 5] = -np.inf
    begin, c = np.array([1, 5, 5, 16]), dc.choices(rng, T, k, X, np.int64)
    w = rng.random((S, X)) + 0.5
    r = dc.balance(z, begin, c, w)
    g = dc.balance_grad(r, 3.0)
    for t in range(T):
        for e in range(X):
            if r["source"][t] < 0:
                assert np.isnan(g[t, e])
                continue
            if not np.isfinite(z[t, e]):
                assert g[t, e] == 0.0
                continue
            d = []
            for h in (1e-4, -1e-4):
                y = z.copy()
                y[t, e] += h
                p = dc.softmax(y)
                sums = np.array([p[r["source"] == s].sum(axis=0) for s in range(S)])
                d.append((r["coef"] * sums).sum())
            assert g[t, e] == pytest.approx(3.0 * (d[0] - d[1]) / 2e-4, rel=1e-6, abs=1e-9)


# ---------------------------------------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------------------------------------

def topology(a2a, n):
    return a2a.Topology(*gen.ring(n)) if n > 1 else a2a.Topology(np.zeros(2, np.int32), np.zeros(0, np.int32))


def logits(rng, tokens, experts, scale=3.0):
    """Rows of every kind that a mask leaves: whole, with some experts left out, one left, none."""
    z = rng.normal(size=(tokens, experts)) * scale + rng.normal(size=experts)
    kind = rng.random(tokens)
    z[rng.random((tokens, experts)) < 0.3 * (kind < 0.3)[:, None]] = -np.inf
    for t in np.flatnonzero(kind > 0.95):
        only = rng.integers(experts)
        z[t, np.arange(experts) != only] = -np.inf
    z[kind > 0.985] = -np.inf
    lowest = (kind > 0.9) & (kind < 0.93)  # a mask of a type's lowest value: the row is one of equals
    z[lowest] = np.where(rng.random((lowest.sum(), experts)) < 0.8, -1e30, z[lowest])
    return z


def rounded(z, type_):
    """z in the type, as a device tensor and in 64 bits."""
    import torch
    with np.errstate(over="ignore"):
        t = torch.from_numpy(np.ascontiguousarray(z)).to(type_)
    return t.cuda(), t.double().numpy()


def check(a2a, S, T, k, X, type_, kind, *, weighted, N=None, seed=0, apart=0, upstream=2.5):
    import torch
    rng = np.random.default_rng(seed + S + T + X)
    N = N or max(S, 2)
    topo = topology(a2a, N)
    begin = dc.begins(kind, S, T, rng)
    ids = np.int64 if (S + T) % 2 else np.int32
    c = dc.choices(rng, T, k, X, ids)
    whole, z = rounded(np.concatenate([logits(rng, T, X), rng.normal(size=(T, apart))], axis=1), type_)
    z, lg = z[:, :X], whole[:, :X]
    cost = rng.random((S, N)) * 7 + 0.25 if weighted else None
    place = rng.integers(-1, N + 1, X).astype(np.int32) if weighted and seed % 2 == 0 else None
    r = dc.balance(z, begin, c, dc.weights(cost, place, S, X))
    d_begin, d_c = device(begin), device(c)
    w = dict(cost=None if cost is None else device(cost), expert_host=None if place is None else device(place))
    loss = torch.full((2,), -7.0, device="cuda")
    counts = torch.full((S + 1, X), -7, dtype=torch.int32, device="cuda")
    sums = torch.full((S + 1, X), -7.0, device="cuda")
    rows = torch.full((S + 1,), -7, dtype=torch.int32, device="cuda")
    ws = topo.alloc_balance_workspace(S, tokens=T, experts=X)
    ws.random_(0, 255)
    up = torch.full((1,), upstream, device="cuda")
    grad_whole = torch.full_like(whole, -7.0)
    grad = grad_whole[:, :X]
    first = None
    for _ in range(2):
        topo.balance_loss(S, logits=lg, choices=d_c, host_begin=d_begin, loss=loss[:1], counts=counts[:S], prob_sums=sums[:S],
                          rows=rows[:S], workspace=ws, **w)
        topo.balance_loss_grad(S, logits=lg, choices_per_token=k, host_begin=d_begin, counts=counts[:S], rows=rows[:S], upstream=up,
                               grad=grad, **w)
        torch.cuda.synchronize()
        bits = [x.clone() for x in (loss, counts, sums, rows, grad_whole)]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, bits))
        first = bits
        ws.random_(0, 255)
    assert (counts[S] == -7).all() and (sums[S] == -7.0).all() and rows[S] == -7 and loss[1] == -7.0
    assert (grad_whole[:, X:] == -7.0).all()
    assert np.array_equal(counts[:S].cpu().numpy(), r["counts"])
    assert np.array_equal(rows[:S].cpu().numpy(), r["rows"])
    tol = column_tolerance(T)
    got = sums[:S].cpu().numpy().astype(np.float64)
    assert (np.abs(got - r["sums"]) <= tol * r["sums"] + 1e-37 * max(T, 1)).all()
    assert float(loss[0]) == pytest.approx(r["loss"], rel=tol + 4 * EPS, abs=1e-35)
    g = grad.double().cpu().numpy()
    want = dc.balance_grad(r, upstream)
    inside = r["source"] >= 0
    assert (g[~inside] == -7.0).all()
    co = r["coef"][np.maximum(r["source"], 0)]
    dot = (r["p"] * co).sum(axis=1, keepdims=True)
    half = float(torch.finfo(type_).eps) / 2
    least = float(torch.finfo(type_).smallest_normal) * float(torch.finfo(type_).eps)  # a subnormal step
    bound = upstream * r["p"] * (np.abs(co) + dot) * ROW_TOLERANCE * 1.01 + half * np.abs(want) * 1.01 + least
    assert (np.abs(g - want)[inside] <= bound[inside]).all()
    topo.close()


TYPES = ["float32", "bfloat16", "float16"]


def dtype_of(name):
    import torch
    return getattr(torch, name)


@gpu
@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("experts", [1, 2, 7, 8, 9, 16, 24, 32, 60, 64, 72, 100, 128, 160, 200, 256, 264, 384, 405, 512, 768, 1024, 1032,
                                     2047, 2560, 4096])
def test_experts(a2a, experts, type_):
    check(a2a, 5, 203, min(6, experts), experts, dtype_of(type_), "ragged", weighted=True, N=17, seed=experts)


@gpu
@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("kind", ["even", "ragged", "one", "gaps", "past"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 8), (1, 0, 2, 16), (1, 3000, 4, 64), (9, 65, 64, 80), (300, 40, 2, 33), (200, 4100, 8, 128)])
def test_sources(a2a, shape, kind, type_):
    S, T, k, X = shape
    check(a2a, S, T, k, X, dtype_of(type_), kind, weighted=S > 1, seed=1)


@gpu
@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("apart", [1, 3, 8, 56])
def test_rows_apart(a2a, apart, type_):
    check(a2a, 7, 400, 3, 120, dtype_of(type_), "ragged", weighted=True, seed=2, apart=apart)


@gpu
def test_a_long_batch(a2a):
    """More tokens than the smallest pieces take, in three sources and in one."""
    import torch
    for S in (1, 3):
        check(a2a, S, 150001, 2, 8, torch.bfloat16, "ragged", weighted=False, seed=5)


@gpu
def test_many_sources(a2a):
    import torch
    check(a2a, 70000, 3000, 2, 8, torch.float32, "ragged", weighted=False, N=2, seed=6)


@gpu
def test_no_upstream_no_tokens_no_sources(a2a):
    import torch
    topo = topology(a2a, 4)
    f = dict(device="cuda")
    z = torch.randn((50, 12), **f)
    c = torch.randint(0, 12, (50, 2), **f)
    begin = torch.tensor([0, 20, 50], **f)
    loss, counts = torch.full((1,), -7.0, **f), torch.empty((2, 12), dtype=torch.int32, **f)
    sums, rows = torch.empty((2, 12), **f), torch.empty(2, dtype=torch.int32, **f)
    ws = topo.alloc_balance_workspace(2, tokens=50, experts=12)
    outs = dict(loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws)
    topo.balance_loss(2, logits=z, choices=c, host_begin=begin, **outs)
    g1, g2 = torch.empty_like(z), torch.empty_like(z)
    one = torch.ones(1, **f)
    topo.balance_loss_grad(2, logits=z, choices_per_token=2, host_begin=begin, counts=counts, rows=rows, grad=g1)
    topo.balance_loss_grad(2, logits=z, choices_per_token=2, host_begin=begin, counts=counts, rows=rows, upstream=one, grad=g2)
    assert torch.equal(g1, g2) and float(g1.abs().max()) > 0
    topo.balance_loss_grad(2, logits=z, choices_per_token=2, host_begin=begin, counts=counts, rows=rows, grad=z)  # in place
    assert torch.equal(g1, z)
    z.fill_(-torch.inf)  # no row is a token
    topo.balance_loss(2, logits=z, choices=c, host_begin=begin, **outs)
    topo.balance_loss_grad(2, logits=z, choices_per_token=2, host_begin=begin, counts=counts, rows=rows, grad=g1)
    assert float(loss) == 0.0 and not counts.any() and not sums.any() and not rows.any() and not g1.any()
    loss.fill_(-7.0)
    topo.balance_loss(2, logits=z[:0], choices=c[:0], host_begin=torch.zeros(3, dtype=torch.int64, **f), **outs)
    assert float(loss) == 0.0 and not counts.any() and not rows.any()
    loss.fill_(-7.0)
    topo.balance_loss(0, logits=z, choices=c, host_begin=begin[:1], loss=loss, counts=counts[:0], prob_sums=sums[:0], rows=rows[:0],
                      workspace=None)
    assert float(loss) == 0.0
    topo.close()


@gpu
def test_nan_and_infinity_stay_in_their_source(a2a):
    import torch
    topo = topology(a2a, 4)
    for bad in (torch.nan, torch.inf):
        z = torch.randn((40, 24), device="cuda")
        z[7, 3] = bad
        c = torch.randint(0, 24, (40, 2), device="cuda")
        begin = torch.tensor([0, 5, 20, 40], device="cuda")
        loss, counts = torch.empty(1, device="cuda"), torch.empty((3, 24), dtype=torch.int32, device="cuda")
        sums, rows = torch.empty((3, 24), device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
        ws = topo.alloc_balance_workspace(3, tokens=40, experts=24)
        topo.balance_loss(3, logits=z, choices=c, host_begin=begin, loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws)
        grad = torch.zeros_like(z)
        topo.balance_loss_grad(3, logits=z, choices_per_token=2, host_begin=begin, counts=counts, rows=rows, grad=grad)
        assert torch.isnan(loss).all() and torch.isnan(sums[1]).all() and torch.isfinite(sums[[0, 2]]).all()
        assert rows.tolist() == [5, 15, 20] and int(counts.sum()) == 80
        assert torch.isnan(grad[7]).all() and torch.isfinite(grad[torch.arange(40, device="cuda") != 7]).all()
    topo.close()


@gpu
def test_rows_past_32_bits(a2a):
    """Rows whose numbers lie past 2^31 from the first: far apart in a large buffer."""
    import torch
    T, X, apart = 40, 24, 64_000_000
    topo = topology(a2a, 3)
    flat = torch.empty((T - 1) * apart + X, dtype=torch.bfloat16, device="cuda")
    z = flat.as_strided((T, X), (apart, 1))
    z.copy_(torch.randn((T, X), device="cuda", generator=torch.Generator("cuda").manual_seed(4)))
    c = torch.randint(0, X, (T, 2), device="cuda")
    begin = torch.tensor([0, 11, 40], device="cuda")
    res = []
    for lg in (z, z.contiguous()):
        loss, counts = torch.empty(1, device="cuda"), torch.empty((2, X), dtype=torch.int32, device="cuda")
        sums, rows = torch.empty((2, X), device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        ws = topo.alloc_balance_workspace(2, tokens=T, experts=X)
        topo.balance_loss(2, logits=lg, choices=c, host_begin=begin, loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws)
        topo.balance_loss_grad(2, logits=lg, choices_per_token=2, host_begin=begin, counts=counts, rows=rows, grad=lg)
        res.append([loss, counts, sums, rows, lg])
    assert all(torch.equal(a, b) for a, b in zip(*res)) and float(res[0][0]) > 0
    topo.close()


@gpu
def test_refusals(a2a):
    import torch
    topo = topology(a2a, 3)
    S, T, k, X = 3, 10, 2, 8
    f = dict(device="cuda")

    def arguments():
        return dict(logits=torch.zeros((T, X), **f), choices=torch.zeros((T, k), dtype=torch.int64, **f),
                    host_begin=torch.tensor([0, 2, 4, T], **f), loss=torch.full((1,), -7.0, **f),
                    counts=torch.full((S, X), -7, dtype=torch.int32, **f), prob_sums=torch.full((S, X), -7.0, **f),
                    rows=torch.full((S,), -7, dtype=torch.int32, **f), workspace=topo.alloc_balance_workspace(S, tokens=T, experts=X))

    def refused(status=None, **other):
        a = {**arguments(), **other}
        with pytest.raises(a2a.A2AError) as e:
            topo.balance_loss(S, **a)
        assert e.value.status == (a2a.ERR_INVALID_ARG if status is None else status)
        torch.cuda.synchronize()
        assert float(a["loss"][0]) == -7.0

    refused(logits=torch.zeros((T, X), dtype=torch.float64, **f))
    refused(logits=torch.zeros((X, T), **f).t())
    refused(logits=torch.zeros((1, X), **f).expand(T, X))
    refused(logits=torch.zeros((T + 1, X), **f))
    refused(cost=torch.zeros((S, 4), dtype=torch.float64, **f))
    refused(cost=torch.zeros((S, 3), **f))
    refused(expert_host=torch.zeros(X, dtype=torch.int64, **f))
    refused(rows=torch.zeros(S + 1, dtype=torch.int32, **f))
    refused(workspace=None)
    refused(workspace=torch.zeros(1 << 20, dtype=torch.uint8, **f)[8:])
    refused(a2a.ERR_WORKSPACE_TOO_SMALL, workspace=arguments()["workspace"][:-256])
    W = a2a.MOST_EXPERTS + 1
    refused(a2a.ERR_NOT_IMPLEMENTED, logits=torch.zeros((T, W), **f), counts=torch.zeros((S, W), dtype=torch.int32, **f),
            prob_sums=torch.zeros((S, W), **f))
    a = arguments()
    for other in (dict(grad=torch.zeros((T, X), dtype=torch.bfloat16, **f)), dict(grad=torch.zeros((T, X - 1), **f)),
                  dict(upstream=torch.zeros(1, dtype=torch.float64, **f)), dict(choices_per_token=0)):
        with pytest.raises(a2a.A2AError):
            topo.balance_loss_grad(S, **{**dict(logits=a["logits"], choices_per_token=k, host_begin=a["host_begin"], counts=a["counts"],
                                                rows=a["rows"], grad=torch.zeros((T, X), **f)), **other})
    topo.close()


@gpu
def test_replayed_beside_an_eager_graph(a2a):
    """Loss and gradient recorded and replayed on new logits, while a program's own autograd graph of the same logits lives."""
    import torch
    topo = topology(a2a, 6)
    S, T, k, X = 6, 500, 2, 40
    g = torch.Generator("cuda").manual_seed(9)
    leaf = torch.randn((T, X), device="cuda", generator=g, requires_grad=True)
    alive = (leaf * 2).sum()
    z = leaf.detach()
    c = z.topk(k, dim=1).indices
    begin = torch.tensor([0, 100, 100, 180, 333, 490, 500], device="cuda")
    loss, counts = torch.empty(1, device="cuda"), torch.empty((S, X), dtype=torch.int32, device="cuda")
    sums, rows = torch.empty((S, X), device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda")
    grad = torch.empty_like(z)
    ws = topo.alloc_balance_workspace(S, tokens=T, experts=X)

    def call(loss, counts, sums, rows, grad, ws):
        topo.balance_loss(S, logits=z, choices=c, host_begin=begin, loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws)
        topo.balance_loss_grad(S, logits=z, choices_per_token=k, host_begin=begin, counts=counts, rows=rows, grad=grad)

    out = (loss, counts, sums, rows, grad, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(*out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*out)
    for rep in range(4):
        with torch.no_grad():
            leaf.normal_(generator=g)
            c.copy_(z.topk(k, dim=1).indices)
        want = [torch.empty_like(x) for x in out]
        call(*want)
        for x in out:
            x.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out[:5], want[:5])), rep
    alive.backward()
    assert (leaf.grad == 2).all()
    del graph
    topo.close()
