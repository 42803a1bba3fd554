"""What the dispatch functions accept and how their calls are cut (csrc/a2a_dispatch_plan.h, plain host arithmetic), and what
the C entry points refuse without a handle: no device needed."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHECK = r"""
#include <cstdio>
#include "a2a_cost_plan.h"
#include "a2a_dispatch_plan.h"
using namespace a2a_dev;
static int bad = 0;
#define WANT(x, y) do { const long long a = (long long)(x), b = (long long)(y); if (a != b) { ++bad; std::printf("line %d: %s = %lld, not %lld\n", __LINE__, #x, a, b); } } while (0)

int main() {
  const int64_t eight = 8;
  alignas(8) char at[16];
  a2a_routing good{};
  good.tokens = 100;
  good.choices_per_token = 4;
  good.experts = 8;
  good.choices_type = A2A_I64;
  good.choices = at;
  good.choices_stride = 4;
  good.host_begin = &eight;
  a2a_routing r = good;
  WANT(check_routing(3, &r, true), A2A_OK);
  WANT(check_routing(0, &r, true), A2A_OK);
  WANT(check_routing(-1, &r, true), A2A_ERR_INVALID_ARG);
  WANT(check_routing(3, nullptr, true), A2A_ERR_INVALID_ARG);
#define WITH(field, value, status) r = good; r.field = value; WANT(check_routing(3, &r, true), status)
  WITH(tokens, -1, A2A_ERR_INVALID_ARG);
  WITH(tokens, INT32_MAX / 4, A2A_OK);
  WITH(tokens, INT32_MAX / 4 + 1, A2A_ERR_NOT_IMPLEMENTED);
  WITH(choices_per_token, 0, A2A_ERR_INVALID_ARG);
  WITH(choices_per_token, 65, A2A_ERR_INVALID_ARG);
  WITH(choices_per_token, 5, A2A_ERR_INVALID_ARG);  // rows would overlap
  WITH(experts, 0, A2A_ERR_INVALID_ARG);
  WITH(reserved, 1, A2A_ERR_INVALID_ARG);
  WITH(choices_type, A2A_F32, A2A_ERR_INVALID_ARG);
  WITH(choices_type, 5, A2A_ERR_INVALID_ARG);
  WITH(choices_stride, INT64_MAX / 8, A2A_ERR_INVALID_ARG);  // past the address space
  WITH(choices, nullptr, A2A_ERR_INVALID_ARG);
  WITH(choices, at + 4, A2A_ERR_INVALID_ARG);
  WITH(host_begin, nullptr, A2A_ERR_INVALID_ARG);
  WITH(host_begin, (const int64_t*)(at + 4), A2A_ERR_INVALID_ARG);
  WITH(expert_host, (const int32_t*)(at + 2), A2A_ERR_INVALID_ARG);
  r = good;
  r.choices_type = A2A_I32;
  r.choices = at + 4;
  WANT(check_routing(3, &r, true), A2A_OK);
  r = good;
  r.tokens = 0;
  r.choices = nullptr;
  WANT(check_routing(3, &r, true), A2A_OK);
  r = good;
  r.choices = nullptr;
  r.choices_type = 77;
  WANT(check_routing(3, &r, false), A2A_OK);

  for (int type : {A2A_F32, A2A_BF16, A2A_F16}) {
    WANT(check_logits(&good, at, type, 8), A2A_OK);
    WANT(check_logits(&good, at, type, 7), A2A_ERR_INVALID_ARG);
    WANT(check_logits(&good, nullptr, type, 8), A2A_ERR_INVALID_ARG);
    WANT(check_logits(&good, at + 1, type, 8), A2A_ERR_INVALID_ARG);
    WANT(check_logits(&good, at, type, INT64_MAX / 4), A2A_ERR_INVALID_ARG);
  }
  WANT(check_logits(&good, at, A2A_I32, 8), A2A_ERR_INVALID_ARG);
  WANT(check_logits(&good, at, -1, 8), A2A_ERR_INVALID_ARG);
  r = good;
  r.experts = A2A_MOST_EXPERTS;
  WANT(check_logits(&r, at, A2A_F16, A2A_MOST_EXPERTS), A2A_OK);
  r.experts = A2A_MOST_EXPERTS + 1;
  WANT(check_logits(&r, at, A2A_F16, A2A_MOST_EXPERTS + 1), A2A_ERR_NOT_IMPLEMENTED);

  // every token has a workgroup, every piece a place, and no launch is too large
  for (int64_t tokens = 0; tokens <= INT32_MAX; tokens = tokens < 3000 ? tokens + 1 : tokens * 5 / 3) {
    const BalanceCut c = balance_cut(tokens);
    if (c.per < 1 || c.groups * c.per < tokens || (c.groups > 0 && (c.groups - 1) * c.per >= tokens) || c.groups > 65535) ++bad;
    for (int64_t sources : {0, 1, 63, 5000, 4194304}) {
      const BalanceLayout l = balance_layout(sources, tokens, 48);
      const size_t places = (size_t)(c.groups + sources);
      if (l.counts - l.sums < places * 48 * 4 || l.rows - l.counts < places * 48 * 4 || l.terms - l.rows < places * 4 ||
          l.total - l.terms < (size_t)source_cut(sources, tokens, 48).groups * 16 || l.total % 256 != 0) ++bad;
      for (int64_t experts : {1, 48, 300, 4096}) {
        const SourceCut q = source_cut(sources, tokens, experts);
        if (q.across < 1 || kBalanceThreads % q.across != 0 || q.groups < 1 || q.groups > kSourceGroups) ++bad;
      }
    }
  }
  // every source and row has a band or pieces, within the LDS of a workgroup; no launch is too large
  for (int64_t sources = 1; sources <= 4194304; sources = sources * 3 / 2 + 1)
    for (int64_t tokens = 0; tokens <= INT32_MAX / 64; tokens = tokens * 2 + 1)
      for (int64_t k : {1, 2, 8, 64})
        for (int64_t rows : {1, 63, 4096, 4097, 65536, 70001})
          for (bool demand : {false, true}) {
            const DispatchCut c = dispatch_cut(sources, tokens, k, rows, demand);
            const int64_t bands = (sources + c.columns - 1) / c.columns;
            if (c.tile < 1 || (int64_t)c.tile * c.tiles < rows || c.columns > kDispatchColumns || (!demand && c.columns != 1) || c.lds > 131328 ||
                c.threads > kDispatchThreads || c.threads % 64 != 0) ++bad;
            if (c.split ? c.per < 1 || c.lds < (size_t)c.tile * 4 || c.groups / c.tiles * c.per < tokens || c.groups % c.tiles != 0
                        : c.groups != bands * c.tiles || c.lds * 2 < (size_t)c.tile * c.columns * 4) ++bad;
            if (sources * rows < 1ll << 33 && c.groups * c.threads > 0xffffffffll) ++bad;
          }
  // path costs: what a way takes fits LDS and the workspace
  for (int N = 2; N <= 65536; N += N < 9000 ? 7 : 131)
    for (int depth : {1, 7, 16, 17, 100, 253, 254, 5000})
      for (int words : {0, 2, 3, 4, 5, 8})
        for (int sources : {1, 63, 64, 512, 513, N}) {
          const CostWay way = cost_way(N, words, depth, sources);
          const CostLayout l = cost_layout(N, words, depth, sources);
          const int nodes = cost_nodes(N, words, depth);
          bool ok = (way == CostWay::kLevels) == (words == 0 || depth > 253) && l.total >= 256 && l.total % 256 == 0;
          if (way != CostWay::kLevels) ok = ok && l.lists - l.prices >= (size_t)N * words * 16;
          if (way == CostWay::kSources)
            ok = ok && nodes > 0 && cost_threads(N, nodes) <= 1024 && cost_threads(N, nodes) * nodes >= N && cost_lds(N, nodes, depth) <= kSmallLds &&
                 (cost_list_in_lds(nodes) || l.picked - l.lists >= (size_t)256 * N * 4) && N <= 65535;
          if (way == CostWay::kScan)
            ok = ok && nodes == 16 && N <= 16384 && cost_scan_lds(N, true) <= kSmallLds && cost_scan_lds(N, false) + 16 <= kSmallLds &&
                 l.picked - l.lists >= (size_t)256 * N * 4 && l.total - l.picked >= 128;
          if (way == CostWay::kScanMemory || way == CostWay::kLevelLaunches) ok = ok && cost_scan_lds(N, false) <= kSmallLds;
          if (way == CostWay::kLevelLaunches) {
            const size_t pairs = (size_t)(sources < 512 ? sources : 512) * N;
            ok = ok && l.masks - l.levels >= pairs && l.pairs - l.masks >= 2 * pairs && l.total - l.pairs >= 16 * pairs;
          }
          if (!ok && ++bad < 10) std::printf("path costs: N %d depth %d words %d sources %d\n", N, depth, words, sources);
        }
  std::printf("%d bad\n", bad);
  return bad != 0;
}
"""


def test_arguments_and_cuts(tmp_path):
    src = tmp_path / "check.cpp"
    src.write_text(CHECK)
    exe = tmp_path / "check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2309_13541_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stdout


@pytest.fixture(scope="module")
def a2a():
    import paper_2309_13541_amd as lib
    if not os.path.exists(lib.library_path()):
        lib.build_library()
    lib.load_library()
    return lib


def test_no_handle(a2a):
    lib, r = a2a.load_library(), a2a.Routing()
    assert lib.a2a_path_costs(None, 0, 1, None, None, None, None, None, 0, None) == a2a.ERR_INVALID_ARG
    assert lib.a2a_dispatch_counts(None, 1, r, None, None) == a2a.ERR_INVALID_ARG
    assert lib.a2a_dispatch_demand(None, 1, r, 0, None, None) == a2a.ERR_INVALID_ARG
    assert lib.a2a_balance_workspace_bytes(None, 1, 1, 1) == 0
    assert lib.a2a_balance_loss(None, 1, r, None, 0, 0, None, None, None, None, None, None, 0, None) == a2a.ERR_INVALID_ARG
    assert lib.a2a_balance_loss_grad(None, 1, r, None, 0, 0, None, None, None, None, None, 0, None) == a2a.ERR_INVALID_ARG


def test_routing_struct_matches_header(a2a):
    import re
    text = open(os.path.join(ROOT, "include", "a2a_topo.h")).read()
    body = re.search(r"typedef struct a2a_routing \{(.*?)\} a2a_routing;", text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert re.findall(r"\b(\w+);", body) == [n for n, _ in a2a.Routing._fields_]
    assert ctypes.sizeof(a2a.Routing) == 56
