"""Timing cases of the expert-dispatch operators: the all-to-all of a mixture-of-experts layer on a direct-connect topology.

Tokens lie on hosts (those of host s are host_begin[s] .. host_begin[s + 1] - 1), experts lie on hosts too, and a router
has chosen k experts for every token.  The operators, by their entry point:
  "counts"     how many choices of each host's tokens fall on each expert
  "demand"     what each host sends to each other one: the demand matrix of a2a_link_loads_demand
  "loss"       the router's balance loss, its probabilities weighted by what a host pays to reach an expert
  "loss_grad"  the same and its gradient with respect to the logits: a training step's calls
  "paths"      the mean cost of the shortest paths of every pair: the gradient of the link loads' total cost by demand

A case: "call", "hosts", "tokens", "experts", "k" choices a token, "type" of the logits or choices, "once" (a token goes
to a host once, however many of its experts are there), "ragged" (token counts of the hosts differ, some are zero),
"weighted" (the loss has costs) and, for "paths", the topology's "family" with "dims" or "d" links a node, links "off"
and the number of "sources".
"""
import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32, "i64": torch.int64}
CHUNK = 1 << 26  # (source, node) pairs or (source, link) pairs that the dense forms take at a time


def _routed(name, call, hosts, tokens, experts, k, type_, *, once=False, ragged=False, weighted=False):
    return {"name": name, "call": call, "hosts": hosts, "tokens": tokens, "experts": experts, "k": k, "type": type_,
            "once": once, "ragged": ragged, "weighted": weighted}


def _paths(name, family, *, hosts=0, d=0, dims="", off=0, sources=0):
    return {"name": name, "call": "paths", "family": family, "hosts": hosts, "d": d, "dims": dims, "off": off,
            "sources": sources}


def listed():
    return [
        # One decoding step of a pod: a token or two a host.
        _routed("counts_step_64", "counts", 64, 96, 64, 2, "i64"),
        # The counts of a whole training batch on 1024 hosts, as they come from a top-k (64-bit ids).
        _routed("counts_batch_1024", "counts", 1024, 1048576, 256, 8, "i64", ragged=True),
        # Traffic of a prefill batch on an 8x8 torus: many tokens for few pairs of hosts.
        _routed("demand_64", "demand", 64, 65536, 128, 4, "i32", ragged=True),
        # Traffic of 81 hosts, odd in every size, a token sent once to a host that has several of its experts.
        _routed("demand_81_once", "demand", 81, 20011, 405, 6, "i64", once=True, ragged=True),
        # Traffic of a 16x16x16 torus with an expert a host: many pairs of hosts, few tokens for each.
        _routed("demand_4096", "demand", 4096, 524288, 4096, 8, "i32"),
        # A small fine-tuning batch.
        _routed("loss_grad_64", "loss_grad", 64, 1024, 64, 2, "f32", weighted=True),
        # The plain balance loss of one long batch, watched during evaluation.
        _routed("loss_plain", "loss", 1, 131071, 160, 6, "f16"),
        # A training step's batch on 1024 hosts.
        _routed("loss_grad_1024", "loss_grad", 1024, 1048576, 256, 8, "bf16", ragged=True, weighted=True),
        # Prices of links to costs of pairs: a small pod after a link event, a rack-sized torus, all pairs of a
        # generalized Kautz topology, and a device's share of the largest network.
        _paths("paths_torus_8x8", "torus", dims="8x8", off=3),
        _paths("paths_torus_16x16x16", "torus", dims="16x16x16", off=49),
        _paths("paths_kautz_16384", "kautz", hosts=16384, d=4, off=65),
        _paths("paths_random_65536", "random", hosts=65536, d=8, sources=1024),
    ]


def _between(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    call = rng.choice(("counts", "demand", "loss", "loss_grad", "loss_grad", "paths", "paths"))
    if call == "paths":
        family = rng.choice(("torus", "kautz", "random", "random"))
        if family == "torus":
            n = _between(rng, 27, 4096)
            r = rng.choice((2, 3))
            side = max(3, int(round(n ** (1.0 / r))))
            sides = [side] * r
            sides[0] = max(3, side + rng.randint(-2, 1))
            dims = "x".join(str(s) for s in sides)
            n = int(np.prod(sides))
            c = _paths("", family, dims=dims, off=rng.randint(0, 2 * n * r // 100))
        else:
            n, d = _between(rng, 64, 65536), rng.randint(2, 8)
            c = _paths("", family, hosts=n, d=d, off=rng.randint(1, max(1, n * d // 200)) if family == "kautz" else 0)
            most = min(n, (1 << 26) // n)  # of 16384 nodes and more not all sources
            c["sources"] = most if rng.random() < 0.5 else rng.randint(max(1, most // 16), most)
    else:
        hosts, k = _between(rng, 4, 4096), rng.randint(1, 8)
        experts = max(k, _between(rng, 8, 512 if call.startswith("loss") else 4096))
        tokens = _between(rng, 64, 1048576)
        if call.startswith("loss"):
            type_ = rng.choice(("f32", "bf16", "bf16", "f16"))
            tokens = min(tokens, (1 << 28) // experts)
            if rng.random() < 0.25:
                hosts = 1
        else:
            type_ = rng.choice(("i32", "i64"))
        c = _routed("", call, hosts, tokens, experts, k, type_, once=call == "demand" and rng.random() < 0.5,
                    ragged=rng.random() < 0.7, weighted=call.startswith("loss") and rng.random() < 0.6)
    del c["name"]
    return c


# -- inputs ---------------------------------------------------------------------------------------------------------


def _topology(case, seed):
    """Out-neighbour CSR: row pointers and targets."""
    rng = np.random.default_rng(seed)
    if case["family"] == "torus":
        dims = [int(x) for x in case["dims"].split("x")]
        ids = np.arange(int(np.prod(dims)))
        cols, stride = [], 1
        for side in dims:
            x = ids // stride % side
            cols += [ids + ((x + 1) % side - x) * stride, ids + ((x - 1) % side - x) * stride]
            stride *= side
        to = np.stack(cols, axis=1)
    elif case["family"] == "kautz":
        ids = np.arange(case["hosts"])
        to = np.stack([(-case["d"] * ids - j) % case["hosts"] for j in range(1, case["d"] + 1)], axis=1)
    else:
        to = np.stack([rng.permutation(case["hosts"]) for _ in range(case["d"])], axis=1)
    n, d = to.shape
    start = np.repeat(np.arange(n), d)
    to = to.reshape(-1)
    stays = start != to
    out = rng.choice(len(to), case["off"], replace=False)
    stays[out] = False
    start, to = start[stays], to[stays]
    ptr = np.concatenate([[0], np.cumsum(np.bincount(start, minlength=n))])
    return ptr.astype(np.int32), to.astype(np.int32)


def _in_links(ptr, to):
    """[d][N] start node and id of each node's in-links, the node itself and -1 where it has fewer."""
    n = len(ptr) - 1
    start = np.repeat(np.arange(n), np.diff(ptr))
    order = np.argsort(to, kind="stable")
    into = to[order]
    first = np.concatenate([[0], np.cumsum(np.bincount(into, minlength=n))])
    place = np.arange(len(into)) - first[into]
    d = int(place.max()) + 1
    node, link = np.tile(np.arange(n), (d, 1)), np.full((d, n), -1)
    node[place, into] = start[order]
    link[place, into] = order
    return torch.from_numpy(node).cuda(), torch.from_numpy(link).cuda()


def _distances(node, link, sources):
    """Hop distances and path counts of all sources, by dense levels."""
    n = node.shape[1]
    dist = torch.full((sources, n), -1, dtype=torch.int32, device="cuda")
    sigma = torch.zeros((sources, n), dtype=torch.float64, device="cuda")
    for s0 in range(0, sources, max(1, CHUNK // n)):
        D, S = dist[s0:s0 + max(1, CHUNK // n)], sigma[s0:s0 + max(1, CHUNK // n)]
        at = torch.arange(len(D), device="cuda")
        D[at, at + s0] = 0
        S[at, at + s0] = 1
        level = 0
        while True:
            paths = torch.zeros_like(S)
            for j in range(len(node)):
                paths += torch.where((D[:, node[j]] == level) & (link[j] >= 0), S[:, node[j]], 0.0)
            new = (paths > 0) & (D < 0)
            if not bool(new.any()):
                break
            level += 1
            D[new] = level
            S[new] = paths[new]
    return dist, sigma


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = _prepare_paths(case, seed, g) if case["call"] == "paths" else _prepare_routed(case, seed, g)
    if own:
        _prepare_own(state)
    return state


def _prepare_paths(case, seed, g):
    ptr, to = _topology(case, seed)
    node, link = _in_links(ptr, to)
    n = len(ptr) - 1
    sources = case["sources"] or n
    dist, sigma = _distances(node, link, sources)
    # prices of links after some rounds of congestion: most near 1, a few far above
    price = torch.rand(len(to), generator=g, device="cuda", dtype=torch.float64).pow(-0.25)
    return {"case": case, "csr": (ptr, to), "node": node, "link": link, "hosts": n, "sources": sources, "dist": dist,
            "sigma": sigma, "price": price, "levels": int(dist.max())}


def _prepare_routed(case, seed, g):
    hosts, T, X, k = case["hosts"], case["tokens"], case["experts"], case["k"]
    rng = np.random.default_rng(seed)
    share = rng.exponential(size=hosts) * (rng.random(hosts) > 0.03) if case["ragged"] else np.ones(hosts)
    share[0] += 1e-3
    begin = np.concatenate([[0], np.round(np.cumsum(share) / share.sum() * T)]).astype(np.int64)
    s = {"case": case, "hosts": hosts, "experts": X, "k": k, "host_begin": torch.from_numpy(begin).cuda(),
         "expert_host": torch.from_numpy(rng.permutation(max(X, hosts))[:X].astype(np.int32) % hosts).cuda()}
    if case["call"].startswith("loss"):
        type_ = TYPES[case["type"]]
        z = torch.randn((T, X), generator=g, device="cuda", dtype=torch.float32)
        z += torch.randn(X, generator=g, device="cuda")  # experts are not equally liked
        z[:, int(rng.integers(X))] = -torch.inf  # one is out of service
        s["choices"] = z.topk(k, dim=1).indices
        z[torch.rand(T, generator=g, device="cuda") < 0.02] = -torch.inf  # padded tokens
        s["logits"] = z.to(type_)
        s["cost"] = None
        if case["weighted"]:
            s["cost"] = 1.0 + 7.0 * torch.rand((hosts, hosts), generator=g, device="cuda", dtype=torch.float64)
        # the loss's share of the total one; half precision has a loss scale
        s["upstream"] = torch.full((1,), 0.01 * (65536.0 if case["type"] == "f16" else 1.0), device="cuda")
    else:
        first = (torch.rand(T, generator=g, device="cuda").pow(1.5) * X).long().clamp_(max=X - 1)
        step = 1 + (torch.rand(T, generator=g, device="cuda") * ((X - 1) // k)).long()
        c = (first[:, None] + step[:, None] * torch.arange(k, device="cuda")) % X
        c[torch.rand(T, generator=g, device="cuda") < 0.02] = -1  # padded tokens
        s["choices"] = c.to(TYPES[case["type"]])
    return s


def _prepare_own(s):
    """The handle of the topology, and the buffers that a program keeps for its calls."""
    import paper_2309_13541_amd as a2a
    call, hosts = s["case"]["call"], s["hosts"]

    def buffer(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if call == "paths":
        s["topo"] = a2a.Topology(*s["csr"])
        s["ws"] = s["topo"].alloc_workspace(s["sources"], a2a.WS_COSTS)
        s["out"] = buffer(s["sources"], hosts, dtype=torch.float64)
        return
    ring = np.arange(hosts, dtype=np.int32)
    ptr = np.arange(hosts + 1, dtype=np.int32) if hosts > 1 else np.zeros(2, dtype=np.int32)
    s["topo"] = a2a.Topology(ptr, (ring + 1) % hosts if hosts > 1 else ring[:0])
    T, X = s["case"]["tokens"], s["experts"]
    if call == "demand":
        s["demand"] = buffer(hosts, hosts, dtype=torch.float64)
        return
    s["counts"] = buffer(hosts, X, dtype=torch.int32)
    if call != "counts":
        s["loss"], s["prob_sums"] = buffer(1), buffer(hosts, X)
        s["rows"] = buffer(hosts, dtype=torch.int32)
        s["ws"] = s["topo"].alloc_balance_workspace(hosts, tokens=T, experts=X)
    if call == "loss_grad":
        s["grad"] = torch.empty_like(s["logits"])


# -- one pass -------------------------------------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    topo, call, hosts = s["topo"], s["case"]["call"], s["hosts"]
    if call == "paths":
        topo.path_costs(0, s["sources"], dist=s["dist"], sigma=s["sigma"], link_cost=s["price"], cost=s["out"],
                        workspace=s["ws"])
        return {"cost": s["out"]}
    routing = dict(choices=s["choices"], host_begin=s["host_begin"], experts=s["experts"])
    if call == "counts":
        topo.dispatch_counts(hosts, counts=s["counts"], **routing)
        return {"counts": s["counts"]}
    if call == "demand":
        topo.dispatch_demand(hosts, expert_host=s["expert_host"], once=s["case"]["once"], demand=s["demand"],
                             **routing)
        return {"demand": s["demand"]}
    weights = dict(cost=s["cost"], expert_host=s["expert_host"] if s["cost"] is not None else None)
    topo.balance_loss(hosts, logits=s["logits"], choices=s["choices"], host_begin=s["host_begin"], loss=s["loss"],
                      counts=s["counts"], prob_sums=s["prob_sums"], rows=s["rows"], workspace=s["ws"], **weights)
    out = {"loss": s["loss"], "counts": s["counts"], "prob_sums": s["prob_sums"], "rows": s["rows"]}
    if call == "loss_grad":
        topo.balance_loss_grad(hosts, logits=s["logits"], choices_per_token=s["k"], host_begin=s["host_begin"],
                               counts=s["counts"], rows=s["rows"], upstream=s["upstream"], grad=s["grad"], **weights)
        out["grad"] = s["grad"]
    return out


def _run_plain(s):
    call, hosts, X, k = s["case"]["call"], s["hosts"], s["experts"] if "experts" in s else 0, s.get("k")
    if call == "paths":
        return {"cost": _plain_paths(s)}
    choices, T = s["choices"].long(), s["case"]["tokens"]
    host = torch.searchsorted(s["host_begin"], torch.arange(T, device="cuda"), right=True) - 1
    if call == "counts":
        at = (host[:, None] * X + choices)[choices >= 0]
        return {"counts": torch.bincount(at, minlength=hosts * X).view(hosts, X).int()}
    if call == "demand":
        to = torch.where(choices >= 0, s["expert_host"].long()[choices.clamp(min=0)], -1)
        goes = to >= 0
        if s["case"]["once"]:
            same = to[:, :, None] == to[:, None, :]
            goes &= ~same.tril(-1).any(2)
        at = (to * hosts + host[:, None])[goes]
        return {"demand": torch.bincount(at, minlength=hosts * hosts).view(hosts, hosts).double()}
    z = s["logits"].float()
    top = z.amax(1, keepdim=True)
    some = top > -torch.inf
    p = torch.where(some, torch.exp(z - top), 0.0)
    p = p / p.sum(1, keepdim=True).clamp(min=torch.finfo(torch.float32).tiny)
    rows = torch.bincount(host[some[:, 0]], minlength=hosts)
    at = (host[:, None] * X + choices)[some[:, 0]]
    counts = torch.bincount(at.flatten(), minlength=hosts * X).view(hosts, X)
    sums = torch.zeros((hosts, X), device="cuda").index_add_(0, host, p)
    weight = s["cost"].float()[:, s["expert_host"].long()] if s["cost"] is not None else torch.ones((1, 1), device="cuda")
    coef = weight * counts * (X / (k * rows.sum().clamp(min=1))) / rows.clamp(min=1)[:, None]
    out = {"loss": (coef * sums).sum().view(1), "counts": counts.int(), "prob_sums": sums, "rows": rows.int()}
    if call == "loss_grad":
        c = coef[host]
        out["grad"] = (s["upstream"] * p * (c - (p * c).sum(1, keepdim=True))).to(s["logits"].dtype)
    return out


def _plain_paths(s):
    node, link, price, n = s["node"], s["link"], s["price"], s["hosts"]
    cost = torch.zeros((s["sources"], n), dtype=torch.float64, device="cuda")
    rows = max(1, CHUNK // n)
    for s0 in range(0, s["sources"], rows):
        D, S, C = (x[s0:s0 + rows] for x in (s["dist"], s["sigma"], cost))
        for level in range(1, s["levels"] + 1):
            total = torch.zeros_like(C)
            for j in range(len(node)):
                on = (D[:, node[j]] == level - 1) & (link[j] >= 0)
                total += torch.where(on, S[:, node[j]] * (C[:, node[j]] + price[link[j]]), 0.0)
            C.copy_(torch.where(D == level, total / S, C))
    return cost


def work(case):
    """Inputs read once, outputs written once."""
    if case["call"] == "paths":
        dims = [int(x) for x in case["dims"].split("x")] if case["dims"] else [case["hosts"]]
        n = int(np.prod(dims))
        pairs = float(case["sources"] or n) * n
        links = n * (2 * len(dims) if case["dims"] else case["d"]) - case["off"]
        # a distance and a count in, a cost out; of one shortest-path link an addition, of more than one the mean
        return {"bytes": 20.0 * pairs + 16.0 * links + 4.0 * n, "flops": pairs}
    hosts, T, X, k = case["hosts"], case["tokens"], case["experts"], case["k"]
    size = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}[case["type"]]
    begin = 8.0 * (hosts + 1)
    if case["call"] == "counts":
        return {"bytes": begin + float(T) * k * size + 4.0 * hosts * X, "flops": float(T) * k}
    if case["call"] == "demand":
        return {"bytes": begin + float(T) * k * size + 4.0 * X + 8.0 * hosts * hosts, "flops": float(T) * k}
    cells = float(T) * X
    bytes_ = begin + cells * size + 8.0 * T * k + 8.0 * hosts * X + 4.0 * hosts
    bytes_ += 8.0 * hosts * min(hosts, X) + 4.0 * X if case["weighted"] else 0.0
    if case["call"] == "loss":
        return {"bytes": bytes_, "flops": 4.0 * cells}
    return {"bytes": bytes_ + 2.0 * cells * size, "flops": 11.0 * cells}


# -- from the definitions, in 64 bits -------------------------------------------------------------------------------


def exact(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["call"] == "paths":
        return {"cost": _exact_paths(_prepare_paths(case, seed, g))}
    s = _prepare_routed(case, seed, g)
    hosts, X, k, T = s["hosts"], s["experts"], s["k"], case["tokens"]
    begin, choices = s["host_begin"].cpu().numpy(), s["choices"].cpu().numpy()
    host = np.repeat(np.arange(hosts), np.diff(begin))
    if case["call"] == "counts":
        counts = np.zeros((hosts, X), dtype=np.int64)
        t, j = np.nonzero(choices >= 0)
        np.add.at(counts, (host[t], choices[t, j]), 1)
        return {"counts": counts.astype(np.int32)}
    place = s["expert_host"].cpu().numpy()
    if case["call"] == "demand":
        t, j = np.nonzero(choices >= 0)
        pairs = np.stack([t, place[choices[t, j]]], axis=1)
        if case["once"]:
            pairs = np.unique(pairs, axis=0)
        demand = np.zeros((hosts, hosts))
        np.add.at(demand, (pairs[:, 1], host[pairs[:, 0]]), 1.0)
        return {"demand": demand}
    z = s["logits"].double()
    rest = torch.logsumexp(z, 1)
    token = torch.isfinite(rest)
    z.sub_(torch.where(token, rest, 0.0)[:, None]).exp_()  # an empty row: exp(-inf) = 0
    running = torch.zeros((T + 1, X), dtype=torch.float64, device="cuda")
    torch.cumsum(z, 0, out=running[1:])
    sums = running[s["host_begin"][1:]] - running[s["host_begin"][:-1]]
    del running
    there = token.cpu().numpy()
    rows = np.bincount(host[there], minlength=hosts)
    counts = np.zeros((hosts, X), dtype=np.int64)
    np.add.at(counts, (np.repeat(host[there], k), choices[there].reshape(-1)), 1)
    slope = X * counts / (k * max(1, rows.sum()) * np.maximum(rows, 1)[:, None])
    if s["cost"] is not None:
        slope = slope * s["cost"].cpu().numpy()[:, place]
    slope = torch.from_numpy(slope).cuda()
    out = {"loss": (slope * sums).sum().view(1), "counts": torch.from_numpy(counts).int(), "prob_sums": sums,
           "rows": torch.from_numpy(rows).int()}
    if case["call"] == "loss_grad":
        c = slope[torch.from_numpy(host).cuda()]
        mean = (z * c).sum(1, keepdim=True)
        out["grad"] = z.mul_(c.sub_(mean)).mul_(float(s["upstream"]))
    return out


def _exact_paths(s):
    """Sum of the costs of all shortest paths, by links, over their number."""
    ptr, to = s["csr"]
    start = torch.from_numpy(np.repeat(np.arange(s["hosts"]), np.diff(ptr))).cuda()
    end = torch.from_numpy(to.astype(np.int64)).cuda()
    rows = max(1, CHUNK // len(to))
    cost = torch.zeros((s["sources"], s["hosts"]), dtype=torch.float64, device="cuda")
    for s0 in range(0, s["sources"], rows):
        D, S, C = (x[s0:s0 + rows] for x in (s["dist"], s["sigma"], cost))
        for level in range(s["levels"]):
            on = (D[:, start] == level) & (D[:, end] == level + 1)
            C.index_add_(1, end, torch.where(on, C[:, start] + S[:, start] * s["price"], 0.0))
        C.div_(S.clamp(min=1.0))
    return cost
