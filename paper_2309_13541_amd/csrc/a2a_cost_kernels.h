// Device code of a2a_path_costs.
#pragma once

#include "a2a_kernels.h"

namespace a2a_dev {

struct CostView {
  const int32_t *in_ptr, *in_col, *in_link;
  const int32_t* dist;
  const double* sigma;
  const double* link_cost;
  double* cost;
  int N, sources, depth;
};

constexpr int kCostThreads = 1024;

// A workgroup per source.  Every last link u -> v of a shortest path to v carries sigma(u) of the sigma(v) paths:
//   cost(v) = sum_u sigma(u) (cost(u) + link_cost(u -> v)) / sum_u sigma(u),
// level by level, so that the costs of the level before are there.
static __global__ void __launch_bounds__(kCostThreads) k_path_costs(CostView c) {
  for (int s = blockIdx.x; s < c.sources; s += gridDim.x) {
    const size_t row = (size_t)s * c.N;
    const int32_t* const dist = c.dist + row;
    const double* const sigma = c.sigma + row;
    double* const cost = c.cost + row;
    for (int v = threadIdx.x; v < c.N; v += kCostThreads) cost[v] = 0.0;
    __syncthreads();
    for (int level = 1; level <= c.depth; ++level) {
      for (int v = threadIdx.x; v < c.N; v += kCostThreads) {
        if (dist[v] != level) continue;
        double sum = 0.0, paths = 0.0;
        for (int p = c.in_ptr[v]; p < c.in_ptr[v + 1]; ++p) {
          const int u = c.in_col[p];
          if (dist[u] != level - 1) continue;
          sum += sigma[u] * (cost[u] + (c.link_cost ? c.link_cost[c.in_link[p]] : 1.0));
          paths += sigma[u];
        }
        cost[v] = sum / paths;
      }
      __syncthreads();
    }
  }
}

}  // namespace a2a_dev
