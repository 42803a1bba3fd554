"""Sources and experts up to the last 32-bit number: launches of counts (csrc/a2a_dispatch_plan.h, checked on the host), the search for a
token's source, and counts of more sources than one launch has workgroups for."""
import os
import subprocess

import pytest

import a2a_inputs as gen

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHECK = r"""
#include <cstdio>
#include "a2a_dispatch_plan.h"
using namespace a2a_dev;

// As the device searches: begin[i] is the number of the first token of entry i.  Whether it ends at `want` entries, and reads what there is.
template <typename F>
static bool found(F begin, unsigned entries, long long t, unsigned want) {
  unsigned lo = 0, hi = entries;
  for (int steps = 0; lo < hi; ++steps) {
    if (steps > 8) return false;
    const unsigned part = search_part(lo, hi);
    unsigned whole = 0;
    for (unsigned lane = 0; lane < kSearchParts; ++lane) {
      const unsigned at = search_behind(lo, hi, part, lane) - 1;
      if (at >= hi || at < lo) return false;
      whole += begin(at) <= t && lo + lane * part < hi;
    }
    if (lo + whole * part >= hi) return hi == want;
    lo += whole * part;
    hi = std::min(lo + part, hi) - 1;
  }
  return lo == want;
}

int main() {
  int bad = 0;
  const int64_t most = INT32_MAX;
  for (int64_t sources : {1ll, 255ll, 16777215ll, 16777216ll, 40000000ll, 1073741824ll, 2147483647ll})
    for (int64_t rows : {1ll, 7ll, 16384ll, 65536ll, 65537ll, 4194305ll, 100000000ll, 500000000ll, 2147483647ll})
      for (int64_t k : {1, 8, 64})
        for (int64_t tokens : {int64_t{0}, int64_t{1}, int64_t{16385}, int64_t{1000003}, most / k}) {
          const DispatchCut c = dispatch_cut(sources, tokens, k, rows, false);
          const bool all = c.split ? c.groups % c.tiles == 0 && c.groups / c.tiles * c.per >= tokens
                                   : c.sources >= 1 && c.groups == c.sources * c.tiles;
          if (!all || (int64_t)c.tile * c.tiles < rows || (c.split && c.sources != sources) || c.sources > sources ||
              c.groups * c.threads > 0xffffffffll) {
            if (++bad < 10) std::printf("sources %lld rows %lld tokens %lld k %lld: %lld workgroups\n", (long long)sources, (long long)rows,
                                        (long long)tokens, (long long)k, (long long)c.groups);
          }
        }
  for (unsigned entries : {1u, 2u, 63u, 64u, 65u, 4097u, 262144u, 2147483584u, 2147483585u, 2147483647u, 2147483648u})
    for (unsigned t : {0u, 1u, 62u, 63u, 64u, 4096u, 1073741823u, 2147483520u, 2147483646u, 2147483647u}) {
      if (!found([](unsigned i) { return (long long)i; }, entries, t, std::min(t + 1, entries))) ++bad;
      if (!found([](unsigned i) { return (long long)i + 1; }, entries, t, std::min(t, entries))) ++bad;
      if (!found([t](unsigned) { return (long long)t + 1; }, entries, t, 0)) ++bad;
      if (!found([t](unsigned) { return (long long)t; }, entries, t, entries)) ++bad;
    }
  std::printf("%d bad\n", bad);
  return bad != 0;
}
"""


def test_launches_and_search(tmp_path):
    src = tmp_path / "check.cpp"
    src.write_text(CHECK)
    exe = tmp_path / "check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2309_13541_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stdout


@pytest.mark.gpu
def test_counts_of_more_sources_than_a_launch_has():
    """Groups of one token or none, 33554437 of them: three launches.  Whole numbers: equal."""
    import torch
    import paper_2309_13541_amd as a2a
    topo = a2a.Topology(*gen.ring(3))
    g = torch.Generator("cuda").manual_seed(7)
    S, T, k, X = 2 * 16777215 + 7, 3_000_000, 2, 2
    begin = torch.randint(-5, T + 5, (S + 1,), device="cuda", generator=g).sort().values
    for dtype in (torch.int32, torch.int64):
        c = torch.randint(-1, X + 1, (T, k), device="cuda", generator=g, dtype=dtype)
        counts = torch.full((S + 1, X), -7, dtype=torch.int32, device="cuda")
        topo.dispatch_counts(S, choices=c, host_begin=begin, experts=X, counts=counts[:S])
        source = torch.searchsorted(begin, torch.arange(T, device="cuda"), right=True) - 1
        on = (c >= 0) & (c < X) & (source >= 0)[:, None] & (source < S)[:, None]
        want = torch.bincount((source[:, None] * X + c)[on], minlength=S * X).view(S, X)
        assert torch.equal(counts[:S].long(), want) and (counts[S] == -7).all()
        assert int(want.sum()) > 0.9 * T  # two of four numbers that a choice may be are experts: one choice a token counts
        assert all(int(p.sum()) > 0.4 * T for p in (want[:16777215], want[16777215:2 * 16777215]))
    topo.close()


@pytest.mark.gpu
def test_most_tokens():
    """2^31 - 1 choices, the most there may be: counts, demands, the loss and its gradient, by what is known of them."""
    import torch
    import paper_2309_13541_amd as a2a
    f = dict(device="cuda")
    topo = a2a.Topology(*gen.ring(5))
    T, S, X = 2**31 - 1, 3, 4
    c = torch.arange(T, dtype=torch.int32, **f).view(T, 1)
    c &= 3
    ends = [0, 1_000_000_001, 1_000_000_004, T]
    begin = torch.tensor(ends, **f)
    want = torch.tensor([[(b - e + 3) // 4 - (a - e + 3) // 4 for e in range(X)] for a, b in zip(ends, ends[1:])])
    counts = torch.empty((S, X), dtype=torch.int32, **f)
    topo.dispatch_counts(S, choices=c, host_begin=begin, experts=X, counts=counts)
    assert torch.equal(counts.cpu().long(), want)
    demand = torch.empty((5, S), dtype=torch.float64, **f)
    for once in (False, True):
        topo.dispatch_demand(S, choices=c, host_begin=begin, experts=X, once=once, demand=demand)
        assert torch.equal(demand[:4].cpu(), want.t().double()) and not demand[4].any()
    z = torch.zeros((T, X), dtype=torch.bfloat16, **f)  # probability 1/4: every sum is a whole number of quarters below 2^24
    loss, sums, rows = torch.empty(1, **f), torch.empty((S, X), **f), torch.empty(S, dtype=torch.int32, **f)
    ws = topo.alloc_balance_workspace(S, tokens=T, experts=X)
    topo.balance_loss(S, logits=z, choices=c, host_begin=begin, loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws)
    n = torch.tensor(ends).diff()
    assert torch.equal(counts.cpu().long(), want) and torch.equal(rows.cpu().long(), n)
    assert torch.equal(sums.cpu(), (n.double() / 4).float()[:, None].expand(S, X))
    assert float(loss) == 1.0  # X / n * sum_s (sum_e counts) / rows * rows / 4: all choices
    up = torch.full((1,), float(T), **f)
    topo.balance_loss_grad(S, logits=z, choices_per_token=1, host_begin=begin, counts=counts, rows=rows, upstream=up, grad=z)
    share = want.double() / n[:, None]  # up p (c - mean c) = X / 4 (share - 1/4)
    for s, t in enumerate([0, 1_000_000_000, 1_000_000_001, 1_000_000_003, 1_000_000_004, T - 1]):
        r = share[s // 2] - 0.25
        # six roundings of the coefficient 4 share, two terms' difference, and bfloat16's
        assert ((z[t].cpu().double() - r).abs() <= 8 * 2.0**-24 * 4 + 2.0**-8 * r.abs()).all()
    topo.close()


@pytest.mark.gpu
def test_cells_past_32_bits():
    """More cells than 32 bits count: 600000 groups x 4096 experts, 46600 x 46600 hosts."""
    import torch
    import paper_2309_13541_amd as a2a
    f = dict(device="cuda")
    g = torch.Generator("cuda").manual_seed(11)
    topo = a2a.Topology(*gen.ring(3))
    S, T, k, X = 600_000, 5003, 3, 4096
    begin = torch.randint(0, T + 1, (S + 1,), generator=g, **f).sort().values
    begin[-20:] = T
    begin[:300_000] = 0
    c = torch.randint(-1, X + 1, (T, k), generator=g, **f)
    z = torch.full((T, X), -torch.inf, **f)  # all on one expert: probability 1
    one = torch.randint(0, X, (T,), generator=g, **f)
    z[torch.arange(T, **f), one] = 2.0
    source = torch.searchsorted(begin, torch.arange(T, **f), right=True) - 1
    inside = (source >= 0) & (source < S)
    on = (c >= 0) & (c < X) & inside[:, None]
    cells = (source[:, None] * X + c)[on]
    assert int(cells.max()) > 2**31
    counts = torch.full((S, X), -7, dtype=torch.int32, **f)
    topo.dispatch_counts(S, choices=c, host_begin=begin, experts=X, counts=counts)

    def check():
        assert int(counts.sum(dtype=torch.int64)) == cells.numel()
        at, n = cells.unique(return_counts=True)
        assert torch.equal(counts.view(-1)[at].long(), n)
        assert int((counts != 0).sum()) == at.numel()

    check()
    sums, rows, loss = torch.full((S, X), -7.0, **f), torch.full((S,), -7, dtype=torch.int32, **f), torch.empty(1, **f)
    ws = topo.alloc_balance_workspace(S, tokens=T, experts=X)
    counts.fill_(-7)
    topo.balance_loss(S, logits=z, choices=c, host_begin=begin, loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws)
    check()
    at, n = (source * X + one)[inside].unique(return_counts=True)
    assert torch.equal(sums.view(-1)[at], n.float()) and int((sums != 0).sum()) == at.numel()
    assert torch.equal(rows.long(), torch.bincount(source[inside], minlength=S))
    del counts, sums, ws
    topo.close()
    N = 46600
    topo = a2a.Topology(*gen.imase_itoh(N, 8))
    begin = torch.linspace(0, T, N + 1, **f).long()
    begin[-1] = T
    c = torch.randint(-1, N + 1, (T, k), generator=g, **f)
    demand = torch.full((N, N), -7.0, dtype=torch.float64, **f)
    topo.dispatch_demand(N, choices=c, host_begin=begin, experts=N, demand=demand)
    source = torch.searchsorted(begin, torch.arange(T, **f), right=True) - 1
    at, n = (c * N + source[:, None])[(c >= 0) & (c < N)].unique(return_counts=True)
    assert int(at.max()) > 2**31
    assert torch.equal(demand.view(-1)[at], n.double()) and int((demand != 0).sum()) == at.numel()
    topo.close()
