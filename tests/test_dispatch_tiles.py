"""Counts and demands whose rows take more than one tile of a workgroup's cells: a shorter last tile, tiles of bands with more than 65535
choices (cells of 32 bits, two halves a tile), tiles of the split form.  Whole numbers: equal."""
import os
import subprocess

import pytest

import a2a_inputs as gen

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
gpu = pytest.mark.gpu

# hosts (0: counts), sources, tokens, k, experts, split, columns, tokens of the heaviest source
CASES = [
    (4097, 4097, 30011, 3, 4097, False, 16, 0), (5000, 5000, 60000, 2, 777, False, 16, 0), (5000, 5000, 60000, 4, 9000, False, 16, 50000),
    (8191, 2100, 20000, 5, 12000, False, 16, 18000), (9000, 2104, 20000, 5, 9000, False, 8, 18000),
    (70001, 300, 4000, 2, 70001, False, 2, 0), (70001, 7, 20000, 4, 3000, False, 1, 19000),
    (20000, 3, 30000, 4, 20000, True, 1, 0), (16385, 1, 40001, 6, 50, True, 1, 0), (40000, 200, 600000, 6, 40000, True, 1, 300000),
    (0, 5, 2000, 3, 70001, False, 1, 0), (0, 40, 200000, 3, 131073, False, 1, 199000), (0, 300, 100000, 4, 66000, False, 1, 99000),
    (0, 3, 30000, 4, 40000, True, 1, 0), (0, 1, 100003, 8, 16385, True, 1, 0), (0, 300, 11500000, 8, 16385, True, 1, 0),
]


def test_cuts_of_the_cases(tmp_path):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include <cstdio>\n#include "a2a_dispatch_plan.h"\nint main() {\n' + "".join(
        f"  {{ const auto c = a2a_dev::dispatch_cut({s}, {t}, {k}, {n or x}, {str(n > 0).lower()}); "
        f'if (c.tiles < 2 || c.split != {str(split).lower()} || c.columns != {columns}) {{ std::printf("{(n, s, t, k, x)}: '
        f'%d tiles, split %d, %d columns\\n", c.tiles, c.split, c.columns); return 1; }} }}\n'
        for n, s, t, k, x, split, columns, _ in CASES) + "  return 0;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2309_13541_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stdout


@gpu
@pytest.mark.parametrize("wide", [False, True], ids=["int32", "int64"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_against_bincount(case, wide):
    import torch
    import paper_2309_13541_amd as a2a
    print(f"case {case}", flush=True)
    N, S, T, k, X, _, _, heavy = case
    f = dict(device="cuda")
    g = torch.Generator("cuda").manual_seed(T + k)
    topo = a2a.Topology(*(gen.imase_itoh(N, 8) if N else gen.ring(3)))  # few levels: quickly made
    c = torch.randint(-1, X + 1, (T, k), generator=g, dtype=torch.int64 if wide else torch.int32, **f)
    cuts = torch.randint(0, T - heavy + 1, (S - 1,), generator=g, **f).sort().values
    cuts[S // 2:] += heavy  # what one source in the middle has besides
    begin = torch.cat([torch.tensor([min(7, T)], **f), cuts.clamp(min=7), torch.tensor([T], **f)])
    source = torch.searchsorted(begin, torch.arange(T, **f), right=True) - 1
    on = (c >= 0) & (c < X) & (source >= 0)[:, None]
    if not N:
        counts = torch.full((S + 2, X), -7, dtype=torch.int32, **f)
        topo.dispatch_counts(S, choices=c, host_begin=begin, experts=X, counts=counts[1:-1])
        want = torch.bincount((source[:, None] * X + c)[on], minlength=S * X).view(S, X)
        assert torch.equal(counts[1:-1].long(), want) and (counts[[0, -1]] == -7).all()
        topo.close()
        return
    place = torch.randint(-2, N + 3, (X,), generator=g, dtype=torch.int32, **f) if X != N else None
    to = torch.where(on, c.long(), 0)
    to = torch.where(on, to if place is None else place[to].long(), -1)
    goes = (to >= 0) & (to < N)
    again = torch.zeros_like(goes)
    for j in range(1, k):
        again[:, j] = ((to[:, :j] == to[:, j:j + 1]) & goes[:, :j]).any(1)
    demand = torch.empty((N + 2, S), dtype=torch.float64, **f)
    for once in (False, True):
        demand.fill_(-7.0)
        topo.dispatch_demand(S, choices=c, host_begin=begin, experts=X, expert_host=place, once=once, demand=demand[1:-1])
        count = goes & ~again if once else goes
        want = torch.bincount((to * S + source[:, None])[count], minlength=N * S).view(N, S)
        assert torch.equal(demand[1:-1], want.double()) and (demand[[0, -1]] == -7.0).all()
    topo.close()
