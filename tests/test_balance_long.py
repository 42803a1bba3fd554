"""Balance loss and gradient of batches long enough that a lane takes several rows of a source one after the other, of every shape that a row
has in lanes: which row comes next, the one asked for ahead, an odd and an even number of them, rows and choices apart.  Against the
definition in 64 bits on the device.

Tolerances, counted before the first run, by what each row has: u = 2^-24 is a rounding.  exp(z - top) is off by 2.22 d + 2 of them, d =
top - z: one of the difference, one of the product with log2(e) and 0.22 for that constant, of d (taken from base 2 to e: the instruction's
argument is 1.44 d, and what it is off by counts ln 2 times), and the instruction's own last bit, 2.  A row's sum is off by the mean of
that over its probabilities, S, and by its additions, A = numbers of a lane + steps between lanes; its reciprocal by 2.  So a probability
is off by 2.22 d + 2 + S + A + 2.  A column's sum adds a rounding for each row of a lane, 6 steps between a wave's rows, 3 between waves, and
the last one.  The mean of a row's coefficients adds A + 4 to each term: the coefficient itself, the multiplication, the reciprocal again.
A gradient adds 4: the product with the reciprocal, the difference, the product, and one to spare for what is small of second order,
which 1 % more covers too.  exp is 0 below 2^-126."""
import os
import subprocess

import numpy as np
import pytest

import a2a_inputs as gen

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
gpu = pytest.mark.gpu
U = 2.0 ** -24

# experts, whether rows are whole pieces of 16 bytes, lanes of a row, numbers of a lane, tokens, choices, sources
CASES = [
    (8, True, 1, 8, 1100003, 2, 5), (16, True, 2, 8, 620009, 3, 40), (32, True, 4, 8, 300007, 5, 1), (64, True, 8, 8, 150001, 9, 7),
    (128, True, 16, 8, 60013, 20, 300), (160, True, 8, 24, 60013, 6, 1), (256, True, 16, 16, 60013, 8, 900),
    (320, True, 8, 40, 60013, 64, 3), (384, True, 16, 24, 33331, 4, 2), (512, True, 16, 32, 33331, 4, 11), (640, True, 16, 40, 33331, 4, 1),
    (1024, True, 16, 64, 33331, 8, 3), (2048, True, 64, 64, 20011, 6, 2),
    (101, False, 16, 8, 60013, 6, 9), (405, False, 16, 32, 33331, 17, 1), (1001, False, 64, 64, 20011, 3, 5),
]


def per_of(tokens):
    """Tokens of a workgroup: csrc/a2a_dispatch_plan.h, balance_cut."""
    return max(16, -(-tokens // 1536), min(256, -(-tokens // 512)))


def test_lanes_take_several_rows(tmp_path):
    """That the cases are what they are meant for: shape of a row as the library chooses it, three rows a lane or more."""
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include <cstdio>\n#include "a2a_dispatch_plan.h"\nusing namespace a2a_dev;\nint main() {\n  int bad = 0;\n' + "".join(
        f"  by_row({X}, {str(wide).lower()}, [&](auto shape) {{ using S = decltype(shape); "
        f"bad += S::kLanes != {lanes} || S::kValues != {values} || balance_cut({T}).per != {per_of(T)} || "
        f"balance_cut({T}).per <= 2 * kBalanceThreads / S::kLanes; }});\n" for X, wide, lanes, values, T, _, _ in CASES)
        + '  std::printf("%d bad\\n", bad);\n  return bad != 0;\n}\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2309_13541_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stdout


def check(case, type_, *, apart=0, grad_apart=0, choices_apart=0, in_place=False, weighted=True, one_source_has_most=False,
          shape=None):
    import torch
    import paper_2309_13541_amd as a2a
    X, _, lanes, values, T, k, S = case
    lanes, values = shape or (lanes, values)
    print(f"case {case} {type_} {apart} {grad_apart} {choices_apart} {in_place}", flush=True)
    dtype, f = getattr(torch, type_), dict(device="cuda")
    g = torch.Generator("cuda").manual_seed(X + S)
    N = max(S, 3)
    topo = a2a.Topology(*gen.ring(N))
    z = torch.randn((T, X + apart), generator=g, **f) * 3 + torch.randn(X + apart, generator=g, **f)
    kind = torch.rand(T, generator=g, **f)
    z[(torch.rand((T, X + apart), generator=g, **f) < 0.3) & (kind < 0.2)[:, None]] = -torch.inf
    z[kind > 0.97] = -torch.inf
    logits = z.to(dtype)[:, :X]
    del z
    c = torch.randint(-1, X + 1, (T, k + choices_apart), generator=g, dtype=torch.int64 if X % 16 == 0 else torch.int32, **f)[:, choices_apart // 2:][:, :k]
    cuts = torch.randint(5, T - 3, (S - 1,), generator=g, **f).sort().values
    if one_source_has_most and S > 2:
        cuts[0], cuts[1:] = 70, T - 40 + torch.arange(S - 2, **f).clamp(max=30)
    begin = torch.cat([torch.tensor([5], **f), cuts, torch.tensor([T - 3], **f)])
    cost = torch.rand((S, N), generator=g, dtype=torch.float64, **f) * 7 + 0.25 if weighted else None
    place = torch.randint(-1, N + 1, (X,), generator=g, dtype=torch.int32, **f) if weighted else None
    up = torch.full((1,), float(T), **f)
    whole = logits.clone() if in_place else torch.full((T, X + grad_apart), -7.0, dtype=dtype, **f)
    ws = topo.alloc_balance_workspace(S, tokens=T, experts=X)
    w = dict(cost=cost, expert_host=place)
    first = None
    for _ in range(2):
        loss, counts = torch.full((1,), -7.0, **f), torch.full((S, X), -7, dtype=torch.int32, **f)
        sums, rows = torch.full((S, X), -7.0, **f), torch.full((S,), -7, dtype=torch.int32, **f)
        ws.random_(0, 255)
        grad = whole.clone()[:, :X] if in_place else whole[:, :X].fill_(-7.0)
        read = grad if in_place else logits
        topo.balance_loss(S, logits=read, choices=c, host_begin=begin, loss=loss, counts=counts, prob_sums=sums, rows=rows, workspace=ws, **w)
        topo.balance_loss_grad(S, logits=read, choices_per_token=k, host_begin=begin, counts=counts, rows=rows, upstream=up, grad=grad, **w)
        bits = [loss, counts, sums, rows, grad.clone()]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, bits))
        first = bits
    assert in_place or (whole[:, X:] == -7.0).all()

    # the definition
    z = logits.double()
    top = z.amax(1, keepdim=True)
    token = top[:, 0] > -torch.inf
    d = torch.where(torch.isfinite(z), top - z, 0.0)
    x = torch.where(token[:, None], torch.exp(z - torch.where(token[:, None], top, 0.0)), 0.0)
    p = x / x.sum(1, keepdim=True).clamp(min=1e-300)
    del x, z, top
    source = torch.searchsorted(begin, torch.arange(T, **f), right=True) - 1
    inside = (source >= 0) & (source < S)
    at = torch.where(inside, source, 0)
    counted = inside & token
    want_rows = torch.bincount(at[counted], minlength=S)
    on = (c >= 0) & (c < X) & counted[:, None]
    want_counts = torch.bincount((at[:, None] * X + c)[on], minlength=S * X).view(S, X)
    assert torch.equal(rows.long(), want_rows) and torch.equal(counts.long(), want_counts)

    additions = values + int(np.log2(lanes))
    off = 2.22 * d + 2  # of an exponential
    off += (p * off).sum(1, keepdim=True) + additions + 2  # of a probability
    of_source = (source == torch.arange(S, **f)[:, None]).double()
    want_sums = of_source @ p
    rows_a_lane = -(-per_of(T) * lanes // 256)
    tol = 1.01 * U * (of_source @ (p * off) + want_sums * (rows_a_lane + 10)) + 2.0 ** -126 * T
    del of_source
    assert ((sums.double() - want_sums).abs() <= tol).all()
    weight = torch.ones((S, X), dtype=torch.float64, **f)
    if weighted:
        there = (place >= 0) & (place < N)
        weight = torch.where(there, cost[:, torch.where(there, place, 0).long()], 0.0)
    coef = X * weight * want_counts / (k * want_rows.sum() * want_rows.clamp(min=1)[:, None])
    want_loss = float((coef * want_sums).sum())
    assert abs(float(loss[0]) - want_loss) <= float((coef * tol).sum()) + 1.01 * U * want_loss
    assert want_loss > 0

    co = (float(T) * coef)[at]
    dot = (p * co).sum(1, keepdim=True)
    want = p * (co - dot)
    dot_off = (p * co * (off + additions + 4)).sum(1, keepdim=True)
    half = float(torch.finfo(dtype).eps) / 2
    least = float(torch.finfo(dtype).smallest_normal) * float(torch.finfo(dtype).eps)
    bound = 1.01 * (U * p * (co + dot_off + (co - dot).abs()) + U * want.abs() * (off + 4) + half * want.abs()) + least + 2.0 ** -126 * (co + dot)
    got = first[4].double()
    assert ((got - want).abs() <= bound)[inside].all()
    assert torch.equal(first[4][~inside], logits[~inside]) if in_place else (got[~inside] == -7.0).all()
    assert not got[inside & ~token].any()
    topo.close()


@gpu
@pytest.mark.parametrize("type_", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_long(case, type_):
    check(case, type_, weighted=case[0] != 64)


@gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rows_apart(case):
    """Logits, gradient and choices as columns of wider matrices, each apart in its own way, whole pieces still; then not."""
    wide = 8 if case[1] else 1
    check(case, "bfloat16", apart=5 * wide, grad_apart=2 * wide, choices_apart=3)
    check(case, "float32", apart=4 if case[1] else 2, grad_apart=12, choices_apart=1)
    if case[0] in (64, 512):  # whole pieces no longer: a number at a time
        check(case, "float16", apart=3, grad_apart=8, shape=(16, 8) if case[0] == 64 else (16, 32))


@gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_in_place(case):
    check(case, "bfloat16", in_place=True)


@gpu
@pytest.mark.parametrize("case", [c for c in CASES if c[6] > 2], ids=str)
def test_one_source_has_most_tokens(case):
    check(case, "float32", one_source_has_most=True)
