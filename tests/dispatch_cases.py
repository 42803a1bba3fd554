"""Inputs of the dispatch tests, and the operators in 64 bits from their definitions (numpy, no device)."""
import numpy as np


def begins(kind, sources, tokens, rng):
    """host_begin of some kind."""
    if kind == "even":
        return np.linspace(0, tokens, sources + 1).round().astype(np.int64)
    if kind == "ragged":  # some sources empty, the first and the last among them where there are enough
        cuts = np.sort(rng.integers(0, tokens + 1, sources - 1))
        b = np.concatenate([[0], cuts, [tokens]])
        if sources > 3:
            b[1], b[-2] = 0, tokens
        return b.astype(np.int64)
    if kind == "one":  # one source has them all
        b = np.zeros(sources + 1, dtype=np.int64)
        b[sources // 2 + 1:] = tokens
        return b
    if kind == "gaps":  # tokens before the first source and behind the last, and an end past the last token
        b = np.linspace(tokens // 5, tokens - tokens // 4, sources + 1).round().astype(np.int64)
        return b
    if kind == "past":  # from before the first token to past the last
        b = np.linspace(-3, tokens + 5, sources + 1).round().astype(np.int64)
        return b
    raise ValueError(kind)


def sources_of(begin, tokens):
    """Source of each token, -1 for those of none."""
    s = np.searchsorted(begin, np.arange(tokens), side="right") - 1
    s[s >= len(begin) - 1] = -1
    return s


def choices(rng, tokens, k, experts, dtype, wild=True):
    c = rng.integers(0, experts, (tokens, k))
    if wild and c.size:
        bad = np.array([-1, -2**31, experts, 2**31 - 1] + ([2**40, -2**40 + 1, 2**32] if dtype == np.int64 else []))
        at = rng.random(c.shape) < 0.1
        c[at] = rng.choice(bad, at.sum())
    return c.astype(dtype)


def counts(begin, c, experts):
    out = np.zeros((len(begin) - 1, experts), dtype=np.int64)
    for s, row in zip(sources_of(begin, len(c)), c):
        if s >= 0:
            for e in row:
                if 0 <= e < experts:
                    out[s, e] += 1
    return out


def demand(begin, c, experts, place, hosts, once):
    out = np.zeros((hosts, len(begin) - 1))
    for s, row in zip(sources_of(begin, len(c)), c):
        if s < 0:
            continue
        to = [int(place[e]) if place is not None else int(e) for e in row if 0 <= e < experts]
        to = [h for h in to if 0 <= h < hosts]
        for h in set(to) if once else to:
            out[h, s] += 1
    return out


def weights(cost, place, sources, experts):
    if cost is None:
        return np.ones((sources, experts))
    h = np.arange(experts) if place is None else np.asarray(place, dtype=np.int64)
    there = (h >= 0) & (h < cost.shape[1])
    return np.where(there, cost[:, np.where(there, h, 0)], 0.0)


def softmax(z):
    """In 64 bits; a row of -inf gives zeroes."""
    with np.errstate(invalid="ignore", over="ignore"):
        top = z.max(axis=1, keepdims=True)
        x = np.exp(z - np.where(top == -np.inf, 0.0, top))
        total = x.sum(axis=1, keepdims=True)
        return np.where(total == 0.0, 0.0, x / np.where(total == 0.0, 1.0, total))


def balance(z, begin, c, weight):
    """p, source of each token (-1: none, or an empty row), counts, prob_sums, rows, coefficients c[s][e], loss."""
    T, X = z.shape
    S = len(begin) - 1
    p = softmax(z)
    s = sources_of(begin, T)
    empty = (z == -np.inf).all(axis=1)
    s_in = np.where(empty, -1, s)
    counts_ = np.zeros((S, X), dtype=np.int64)
    sums, rows = np.zeros((S, X)), np.zeros(S, dtype=np.int64)
    for t in range(T):
        if s_in[t] >= 0:
            sums[s[t]] += p[t]
            rows[s[t]] += 1
            for e in c[t]:
                if 0 <= e < X:
                    counts_[s[t], e] += 1
    n, k = rows.sum(), c.shape[1]
    coef = X * weight * counts_ / (k * max(n, 1) * np.maximum(rows, 1)[:, None])
    return dict(p=p, source=s, counts=counts_, sums=sums, rows=rows, coef=coef, loss=float((coef * sums).sum()))


def balance_grad(r, upstream=1.0):
    """d loss / d logits, with the choices as they are; NaN for tokens of no source (they are not written)."""
    c = r["coef"][np.maximum(r["source"], 0)]
    g = upstream * r["p"] * (c - (r["p"] * c).sum(axis=1, keepdims=True))
    g[r["source"] < 0] = np.nan
    return g


def path_costs(row_ptr, col, dist, sigma, link_cost):
    """By levels, each link's share of the paths through it."""
    start = np.repeat(np.arange(len(row_ptr) - 1), np.diff(row_ptr))
    total = np.zeros(dist.shape)
    for level in range(int(dist.max(initial=0))):
        for u, v, w in zip(start, col, link_cost):
            on = (dist[:, u] == level) & (dist[:, v] == level + 1)
            total[on, v] += total[on, u] + sigma[on, u] * w
    return np.where(sigma > 0, total / np.maximum(sigma, 1), 0.0)
