// How a call of a2a_path_costs is cut up: plain host arithmetic, no HIP, so that it can be checked over its whole range
// without a device.
#pragma once

#include "a2a_plan.h"

namespace a2a_dev {

constexpr int kCostThreads = 1024;
constexpr int kCostDeepest = 253;   // levels are bytes, 255 is a node that is not reached, and no level is one less
constexpr int kCostScanNodes = 16;  // nodes of a thread in k_cost_scan
constexpr int kCostGroups = 256;    // workgroups whose lists lie in the workspace

// Nodes of a thread where a source's state fits LDS (k_cost_sources); 0: it does not, or there is no link table.
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

// Topologies of few levels or many nodes: a scan of all nodes a level, of a source by a workgroup or of all sources by a launch.
constexpr int kCostFewLevels = 16;
constexpr int kCostLevelSources = 512;  // at a time, at the most
constexpr int kCostLevelThreads = 256, kCostLevelNodes = 1024;  // of a workgroup
enum class CostWay { kLevels, kSources, kScan, kScanMemory, kLevelLaunches };
constexpr CostWay cost_way(int N, int words, int depth, int sources) {
  if (words == 0 || depth > kCostDeepest) return CostWay::kLevels;
  if (N > kScaledNodes && N <= kCostScanNodes * kCostThreads && depth <= kCostFewLevels) return CostWay::kScan;
  if (cost_nodes(N, words, depth) > 0) return CostWay::kSources;
  return depth <= kCostFewLevels && sources >= 64 ? CostWay::kLevelLaunches : CostWay::kScanMemory;
}
constexpr size_t cost_scan_lds(int N, bool costs) { return (size_t)(N + 15) / 16 * 16 * (costs ? 9 : 1); }

struct CostLayout {
  size_t prices = 0, lists = 0, levels = 0, masks = 0, pairs = 0, total = 0;
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
  const bool lists = way == CostWay::kSources && !cost_list_in_lds(cost_nodes(N, words, depth));
  const size_t marks = way == CostWay::kLevelLaunches ? (size_t)std::min(sources, kCostLevelSources) * N : 0;
  l.prices = part(way != CostWay::kLevels ? (size_t)N * words * 16 : 0);
  l.lists = part(lists ? (size_t)kCostGroups * N * 4 : 0);
  l.levels = part(marks);
  l.masks = part(marks * 2);
  l.pairs = part(marks * 16);
  l.total = off > 0 ? off : 256;
  return l;
}

}  // namespace a2a_dev
