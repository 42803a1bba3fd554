// How a call of a2a_path_costs is cut up: plain host arithmetic, no HIP, so that it can be checked over its whole range
// without a device.
#pragma once

#include "a2a_plan.h"

namespace a2a_dev {

constexpr int kCostThreads = 1024;
constexpr int kCostDeepest = 253;   // levels are bytes, 255 is a node that is not reached, and no level is one less
constexpr int kCostScanNodes = 16;  // nodes of a thread in k_cost_scan
constexpr int kCostGroups = 256;    // workgroups whose lists lie in the workspace

// Nodes of a thread where a source's state fits LDS (k_cost_sources); 0: it does not, or there is no link table.  As many as leave two
// workgroups of a compute unit their registers (16x16x16 torus, 4 or 8 nodes a thread: 208, 251 us).
constexpr int cost_nodes(int N, int words, int depth) {
  if (words == 0 || depth > kCostDeepest) return 0;
  return N <= 1024 ? 2 : N <= 4096 ? 4 : N <= kScaledNodes ? 8 : N <= 16 * kCostThreads ? 16 : 0;
}
constexpr bool cost_list_in_lds(int nodes) { return nodes < 16; }
constexpr int cost_threads(int N, int nodes) {
  const int waves = (N + nodes * kSmallWave - 1) / (nodes * kSmallWave);
  return waves * kSmallWave;
}
// LDS of a source: a double and a level byte a node, its place in the order of levels, starts of the levels.
constexpr size_t cost_lds(int N, int nodes, int depth) {
  const size_t n = (size_t)(N + 15) / 16 * 16;
  return 8 * n + (cost_list_in_lds(nodes) ? 4 * n : 0) + ((size_t)depth + 2 + 3) / 4 * 16 + n;
}
static_assert(cost_lds(16 * kCostThreads, 16, kCostDeepest) <= kSmallLds && cost_lds(kScaledNodes, 8, kCostDeepest) <= kSmallLds);

// How a call goes.  us of 1024 sources by k_cost_scan and k_cost_sources: a generalized Kautz topology of 16000 nodes of degree 2 82, 255
// (no path counts, nothing sorted); random ones, with several last links a node, 16384 of degree 4 423, 263, 9000 of degree 8 257, 233;
// 22x22x22 torus (33 levels) 553, 283.  So both are launched where the levels are few, and k_cost_pick finds out from some
// of the call's sources which of them has something to do (some 15 us: not for few sources).  Of more nodes by launches a level and by k_cost_scan_memory:
// 65536 of degree 8, 64 sources 300, 803, 256 sources 1064, 1433; 20000 of degree 4, 64 sources 97, 171, 256 sources 246, 241;
// 16x16x16x16 torus (32 levels), 256 sources 3060, 2486.
constexpr int kCostPickSources = 512, kCostPicked = 16;
constexpr int kCostFewLevels = 16;
constexpr int kCostLevelSources = 512;  // at a time, at the most
constexpr int kCostLevelThreads = 256, kCostLevelNodes = 1024;  // of a workgroup
enum class CostWay { kLevels, kSources, kScan, kScanMemory, kLevelLaunches };
constexpr CostWay cost_way(int N, int words, int depth, int sources) {
  if (words == 0 || depth > kCostDeepest) return CostWay::kLevels;
  if (N > kScaledNodes && N <= kCostScanNodes * kCostThreads && depth <= kCostFewLevels && sources >= kCostPickSources) return CostWay::kScan;
  if (cost_nodes(N, words, depth) > 0) return CostWay::kSources;
  return depth <= kCostFewLevels && sources >= 64 ? CostWay::kLevelLaunches : CostWay::kScanMemory;
}
constexpr size_t cost_scan_lds(int N, bool costs) { return (size_t)(N + 15) / 16 * 16 * (costs ? 9 : 1); }

struct CostLayout {
  size_t prices = 0, lists = 0, picked = 0, levels = 0, masks = 0, pairs = 0, total = 0;
};
inline CostLayout cost_layout(int N, int words, int depth, int sources) {
  CostLayout l;
  size_t off = 0;
  const auto part = [&off](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  const CostWay way = cost_way(N, words, depth, sources);
  const bool lists = way == CostWay::kScan || (way == CostWay::kSources && !cost_list_in_lds(cost_nodes(N, words, depth)));
  const size_t marks = way == CostWay::kLevelLaunches ? (size_t)std::min(sources, kCostLevelSources) * N : 0;
  l.prices = part(way != CostWay::kLevels ? (size_t)N * words * 16 : 0);
  l.lists = part(lists ? (size_t)kCostGroups * N * 4 : 0);
  l.picked = part(way == CostWay::kScan ? kCostPicked * 8 : 0);
  l.levels = part(marks);
  l.masks = part(marks * 2);
  l.pairs = part(marks * 16);
  l.total = off > 0 ? off : 256;
  return l;
}

}  // namespace a2a_dev
