// Device code of a2a_path_costs.
//
// A last link u -> v of a shortest path to v carries sigma(u) of its sigma(v) paths, so with C(v) = sigma(v) cost(v), the
// costs of all shortest paths to v together,
//   C(v) = B(v) + sum_u C(u),  B(v) = sum_u sigma(u) link_cost(u -> v),
// over the links u -> v with D(u) = D(v) - 1.  B and which links these are need no cost of any other node: all nodes at
// once.  The sums need the level before: level by level.  One reciprocal a node at the end.
#pragma once

#include "a2a_cost_plan.h"
#include "a2a_small_kernels.h"

namespace a2a_dev {

struct CostView {
  const int32_t *in_ptr, *in_col, *in_link;
  const uint32_t* in;  // link table (SmallView), or null
  const int32_t* dist;
  const double* sigma;
  const double* link_cost;
  double* prices;   // [words of the link table][N][2], if there are link costs: those of a wave's nodes lie next to each other
  uint32_t* lists;  // [workgroups][N]
  int* picked;      // null, or [kCostPicked][2] what k_cost_pick has found
  unsigned char* levels;  // [sources][N], with the places of the last links
  uint16_t* masks;
  double2* pairs;  // [sources][N] path count and cost
  double* cost;
  int N, sources, depth, words;
};

// Element i of an array at a uniform address, by a 32-bit offset of bytes: no 64-bit addition a lane.
template <typename T>
__device__ __forceinline__ T& near(T* base, int i) {
  return *reinterpret_cast<T*>(reinterpret_cast<char*>(const_cast<std::remove_const_t<T>*>(base)) + (uint32_t)(i * (int)sizeof(T)));
}
__device__ __forceinline__ int price_at(int place, int v, int N) { return (place / 2 * N + v) * 2 + place % 2; }

// Link costs by place of the link table.
static __global__ void __launch_bounds__(kBlock) k_cost_prices(CostView c) {
  const int places = 2 * c.words;
  const int i = blockIdx.x * kBlock + threadIdx.x;
  if (i >= c.N * places) return;
  const int q = i / 2 / c.N, v = i / 2 - q * c.N, p = c.in_ptr[v] + 2 * q + i % 2;
  c.prices[i] = p < c.in_ptr[v + 1] ? c.link_cost[c.in_link[p]] : 0.0;
}

// Whether more than a sixth of those nodes have several last links: then taking the nodes in order (k_cost_sources) is the faster way.
__device__ __forceinline__ bool in_order(const CostView& c) {
  int reached = 0, several = 0;
  for (int i = 0; i < kCostPicked; ++i) {
    reached += c.picked[2 * i];
    several += c.picked[2 * i + 1];
  }
  return 6 * several > reached;
}

// Lanes whose x, of `bits` bits, is this lane's.
__device__ __forceinline__ uint64_t lanes_like(unsigned x, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot(x >> b & 1u);
    m &= x >> b & 1u ? set : ~set;
  }
  return m;
}

// Waves a SIMD: two workgroups of a compute unit where their nodes' registers allow it.
constexpr int cost_waves(int words, int nodes) { return nodes <= 4 && words <= 4 ? 8 : 4; }

// A workgroup per source, its state in LDS: an array of doubles that holds path counts, then B, then C; a level byte a
// node; the nodes in the order of levels, with a bit for each place of the link table that is a last link.  A thread has
// kNodes nodes for what needs no order.  Places in a level are handed out a wave at a time (an atomic addition a level and
// wave); their order changes nothing, a node's sum is its own.  16x16x16 torus, all sources, 210 us (336 MB; 3.1
// ms with everything in memory): vector ALUs are busy 63 % of the time, LDS about 40 %, with two workgroups a compute unit, all the waves that
// it takes, and barriers between levels.
template <int KS, int kNodes>
__global__ void __launch_bounds__(kCostThreads, cost_waves(KS, kNodes)) k_cost_sources(CostView c) {
  constexpr bool kInLds = cost_list_in_lds(kNodes);
  constexpr int kShift = kNodes < 16 ? 3 : 0;  // ids of the table are 8 x id up to kScaledNodes
  if (c.picked != nullptr && !in_order(c)) return;
  extern __shared__ __align__(16) unsigned char cost_state[];
  const int N = c.N, T = blockDim.x, pad = (N + 15) / 16 * 16;
  double* const value = (double*)cost_state;
  uint32_t* const list = kInLds ? (uint32_t*)(value + pad) : c.lists + (size_t)blockIdx.x * N;
  int* const start = kInLds ? (int*)(value + pad) + pad : (int*)(value + pad);
  unsigned char* const level = (unsigned char*)(start + (c.depth + 2 + 3) / 4 * 4);
  const int bits = 32 - __builtin_clz(c.depth | 1);
  const bool priced = c.link_cost != nullptr;
  for (int s = blockIdx.x; s < c.sources; s += gridDim.x) {
    const size_t row = (size_t)s * N;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // what a thread's nodes need is computed anew for each source: kept, it takes the registers
    constexpr bool kKept = kNodes < 16;  // path counts in registers to the end; read again where they do not fit
    double sigma[kNodes];
    for (int i = tid; i < c.depth + 2; i += T) start[i] = 0;
#pragma unroll
    for (int i = 0; i < kNodes; ++i) {
      const int v = tid + i * T;
      sigma[i] = v < N ? near(c.sigma + row, v) : 0.0;
    }
    for (int v = tid; v < N; v += T) {
      const int d = near(c.dist + row, v);
      level[v] = (unsigned char)((unsigned)d <= (unsigned)c.depth ? d : kSmallUnseen);
    }
#pragma unroll
    for (int i = 0; i < kNodes; ++i) {
      const int v = tid + i * T;
      if (v < N) value[v] = sigma[i];
    }
    __syncthreads();
    const auto level_of = [&](int v) { return v < N ? (int)level[v] : kSmallUnseen; };
    double b[kNodes];
    uint32_t place[kNodes];  // last links above, place in its level below
#pragma unroll
    for (int i = 0; i < kNodes; ++i) {
      const int v = tid + i * T;
      const int l = level_of(v);
      uint32_t mask = 0;
      b[i] = 0.0;
      if (l - 1u < (unsigned)c.depth) {
        SmallRow<KS> r;
        r.load(c.in, 8 * v);
#pragma unroll
        for (int j = 0; j < 2 * KS; ++j) mask |= (level[r.template at<0>(j) >> kShift] + 1 == l ? 1u : 0u) << j;
        if (priced) {
          double2 q[KS];
#pragma unroll
          for (int j = 0; j < KS; ++j) q[j] = near((const double2*)c.prices, j * N + v);
#pragma unroll
          for (int j = 0; j < 2 * KS; ++j) {
            const double paths = value[r.template at<0>(j) >> kShift];
            b[i] = __builtin_fma(mask >> j & 1u ? paths : 0.0, j & 1 ? q[j / 2].y : q[j / 2].x, b[i]);
          }
        } else {
          b[i] = value[v];
        }
      }
      const uint64_t like = lanes_like(l, bits) & __ballot(l != kSmallUnseen);
      int at = 0;
      if (l != kSmallUnseen) {
        const int first = __builtin_ctzll(like);
        if (lane_id() == first) at = atomicAdd(&start[l + 1], __popcll(like));
        at = __shfl(at, first, kWave) + (int)rank_in(like);
      }
      place[i] = mask << 16 | (uint32_t)at;
      __builtin_amdgcn_sched_barrier(0);  // rows of several nodes at a time do not fit the registers
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kNodes; ++i) {
      const int v = tid + i * T;
      if (v < N) value[v] = b[i];
    }
    if (tid < kWave) {  // starts from counts
      int before = 0;
      for (int i0 = 0; i0 < c.depth + 2; i0 += kWave) {
        const int i = i0 + lane_id();
        int x = i < c.depth + 2 ? start[i] : 0;
#pragma unroll
        for (int m = 1; m < kWave; m *= 2) {
          const int y = __shfl_up(x, m, kWave);
          if (lane_id() >= m) x += y;
        }
        x += before;
        if (i < c.depth + 2) start[i] = x;
        before = __shfl(x, kWave - 1, kWave);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kNodes; ++i) {
      const int v = tid + i * T;
      const int l = level_of(v);
      if (l != kSmallUnseen) list[start[l] + (place[i] & 0xffffu)] = (place[i] & 0xffff0000u) | (uint32_t)(v << kShift);
    }
    __syncthreads();
    const auto at = [&](uint32_t id) -> double& { return value[id >> kShift]; };
    const auto add = [&](uint32_t w, const SmallRow<KS>& r) {
      // all in flight together: one by one, where there is a last link, each would wait for the one before
      double x = at(w & 0xffffu), y[2 * KS];
#pragma unroll
      for (int j = 0; j < 2 * KS; ++j) y[j] = at(r.template at<0>(j));
#pragma unroll
      for (int j = 0; j < 2 * KS; ++j) x += w >> (16 + j) & 1u ? y[j] : 0.0;
      at(w & 0xffffu) = x;
    };
    const auto fetch = [&](int i, uint32_t& w, SmallRow<KS>& r) {
      w = list[i];
      r.load(c.in, kShift ? w & 0xffffu : (w & 0xffffu) * 8);
    };
    // a thread's first node of a level is asked for while the level before is worked on
    int i0 = start[1], i1 = start[2];
    uint32_t w = 0;
    SmallRow<KS> r;
    if (i0 + tid < i1) fetch(i0 + tid, w, r);
    for (int d = 1; d <= c.depth && i0 < i1; ++d) {
      const int i2 = d < c.depth ? start[d + 2] : i1;
      uint32_t wn = 0;
      SmallRow<KS> rn;
      if (i1 + tid < i2) fetch(i1 + tid, wn, rn);
      if (i0 + tid < i1) add(w, r);
      for (int i = i0 + tid + T; i < i1; i += T) {
        uint32_t wx;
        SmallRow<KS> rx;
        fetch(i, wx, rx);
        add(wx, rx);
      }
      lds_barrier();
      i0 = i1;
      i1 = i2;
      w = wn;
      r = rn;
    }
#pragma unroll
    for (int i = 0; i < kNodes; ++i) {
      const int v = tid + i * T;
      if (v < N) near(c.cost + row, v) = level[v] - 1u < (unsigned)c.depth ? value[v] * recip(kKept ? sigma[i] : near(c.sigma + row, v)) : 0.0;
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
  }
}

static __device__ const double kCostUnit = 1.0;  // of a link, where the call has no link costs

// Mean over the last links of a node's shortest paths, those that `mask` says, with everything that it takes in flight together:
// a place without such a link asks for what node 0 has.  (Lanes that ask for the same line, and prices next to each other, are one lookup in
// L1: 10 lookups a request of 64 lanes for 65536 nodes of degree 8.)
// of(u): path count and cost of node u.
template <int KS, typename F>
__device__ __forceinline__ double cost_mean(const CostView& c, F&& of, const SmallRow<KS>& r, uint32_t mask, int v) {
  constexpr int kHalf = KS <= 5 ? 2 * KS : KS;  // as many at a time as there are registers for
  static_assert(kHalf % 2 == 0 && 2 * KS % kHalf == 0, "prices come in pairs");
  double sum = 0.0, paths = 0.0;
#pragma unroll
  for (int j0 = 0; j0 < 2 * KS; j0 += kHalf) {
    double2 n[kHalf];
    double w[kHalf];
#pragma unroll
    for (int j = 0; j < kHalf; ++j) {
      n[j] = of(mask >> (j0 + j) & 1u ? r.template at<0>(j0 + j) : 0u);
    }
    if (c.link_cost != nullptr) {
#pragma unroll
      for (int j = 0; j < kHalf; j += 2) {
        const double2 p = near((const double2*)c.prices, (j0 + j) / 2 * c.N + v);
        w[j] = p.x;
        w[j + 1] = p.y;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kHalf; ++j) w[j] = 1.0;
    }
#pragma unroll
    for (int j = 0; j < kHalf; ++j) {
      const bool on = mask >> (j0 + j) & 1u;  // (the node has no cost yet: what is there may be no number)
      sum = __builtin_fma(on ? n[j].x : 0.0, on ? n[j].y + w[j] : 0.0, sum);
      paths += on ? n[j].x : 0.0;
    }
  }
  return sum / paths;
}

template <int KS>
__device__ __forceinline__ uint32_t last_links(const SmallRow<KS>& r, const unsigned char* level, int l) {
  uint32_t mask = 0;
#pragma unroll
  for (int j = 0; j < 2 * KS; ++j) mask |= (level[r.template at<0>(j)] + 1 == l ? 1u : 0u) << j;
  return mask;
}

// The link of `mask`, or the first, and where it starts.
template <int KS>
__device__ __forceinline__ void only_link(const SmallRow<KS>& r, uint32_t mask, int& place, uint32_t& from) {
  place = mask != 0 ? __builtin_ctz(mask) : 0;
  from = r.template at<0>(0);
#pragma unroll
  for (int j = 1; j < 2 * KS; ++j) from = place == j ? r.template at<0>(j) : from;
}

// Nodes that kCostPicked of the call's sources reach, and those of them with several last links: a workgroup a source.
template <int KS>
__global__ void __launch_bounds__(kCostThreads) k_cost_pick(CostView c) {
  extern __shared__ __align__(16) unsigned char cost_state[];
  unsigned char* const level = cost_state;
  int* const found = (int*)(cost_state + (c.N + 15) / 16 * 16);  // reached, with several last links
  if (threadIdx.x < 2) found[threadIdx.x] = 0;
  for (int v = threadIdx.x; v < c.N; v += kCostThreads) {
    const int d = c.dist[(size_t)blockIdx.x * (c.sources / kCostPicked) * c.N + v];
    level[v] = (unsigned char)((unsigned)d <= (unsigned)c.depth ? d : kSmallUnseen);
  }
  __syncthreads();
  int reached = 0, several = 0;
  for (int v = threadIdx.x; v < c.N; v += kCostThreads) {
    const int l = level[v];
    SmallRow<KS> r;
    r.load(c.in, 8 * v);
    const uint32_t mask = last_links(r, level, l);
    reached += l - 1u < (unsigned)c.depth;
    several += l - 1u < (unsigned)c.depth && (mask & (mask - 1)) != 0;
  }
  atomicAdd(&found[0], reached);
  atomicAdd(&found[1], several);
  __syncthreads();
  if (threadIdx.x < 2) c.picked[2 * blockIdx.x + threadIdx.x] = found[threadIdx.x];
}

// A workgroup per source, level bytes and costs in LDS, every level a pass over a thread's nodes; a wave without a node of
// the level goes on.  What a node needs whose shortest paths have one last link, its start and its cost, is found for all
// nodes at once before; path counts are wanted only where there are several.  The next source's distances are under way
// meanwhile.  Where most nodes have one last link: all 16384 sources of a generalized Kautz topology of degree 4 1.25 ms, 3.2 GB without
// the path counts, 2.6 TB/s (costs are written in whole lines, 2.16 GB by the counter).  No unit is full: vector ALUs 44 %, L1 73 % with
// data on its way.  A workgroup of 16 waves is all that LDS has room for, and its phases follow one another.
template <int KS>
__global__ void __launch_bounds__(kCostThreads) k_cost_scan(CostView c) {
  constexpr int kNodes = kCostScanNodes, kAhead = KS <= 4 ? 4 : 1;
  constexpr uint32_t kSeveral = 1u << 31;
  if (in_order(c)) return;
  extern __shared__ __align__(16) unsigned char cost_state[];
  const int N = c.N;
  double* const value = (double*)cost_state;
  unsigned char* const level = cost_state + 8 * ((N + 15) / 16 * 16);
  const bool priced = c.link_cost != nullptr;
  int dist[kNodes];
  const auto ask = [&](int s, int tid) {
#pragma unroll
    for (int i = 0; i < kNodes; ++i) dist[i] = near(c.dist + (size_t)s * N, min(tid + i * kCostThreads, N - 1));
  };
  ask(blockIdx.x, threadIdx.x);
  for (int s = blockIdx.x; s < c.sources; s += gridDim.x) {
    const size_t row = (size_t)s * N;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    uint32_t levels[kNodes / 4] = {};
#pragma unroll
    for (int i = 0; i < kNodes; ++i) {
      const int v = tid + i * kCostThreads;
      const int l = v < N && (unsigned)dist[i] <= (unsigned)c.depth ? dist[i] : kSmallUnseen;
      levels[i / 4] |= (uint32_t)l << (i % 4 * 8);
      if (v < N) {
        level[v] = (unsigned char)l;
        if (l == 0 || l == kSmallUnseen) {
          value[v] = 0.0;
          near(c.cost + row, v) = 0.0;
        }
      }
    }
    __syncthreads();
    uint32_t from[kNodes];
    double price[kNodes];
#pragma unroll
    for (int i0 = 0; i0 < kNodes; i0 += kAhead) {
      asm volatile("" : "+v"(tid));
      SmallRow<KS> r[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) r[i].load(c.in, 8 * min(tid + (i0 + i) * kCostThreads, N - 1));
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int v = min(tid + (i0 + i) * kCostThreads, N - 1);
        const uint32_t mask = last_links(r[i], level, (int)(levels[(i0 + i) / 4] >> ((i0 + i) % 4 * 8) & 0xffu));
        int place;
        only_link(r[i], mask, place, from[i0 + i]);
        if ((mask & (mask - 1)) != 0) from[i0 + i] |= kSeveral;
        asm volatile("" : "+v"(from[i0 + i]));  // here, not where it is used: the row would have to stay
        price[i0 + i] = *(priced ? c.prices + price_at(place, v, N) : &kCostUnit);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("" : "+v"(tid));
    ask(min(s + (int)gridDim.x, c.sources - 1), tid);
    const double* const sigma = c.sigma + row;
    const auto of = [&](uint32_t u) { return make_double2(sigma[u], value[u]); };
    for (int l = 1; l <= c.depth; ++l) {
      asm volatile("" : "+v"(tid));  // nor are places kept from one level to the next
      uint32_t several = 0;  // a bit for each node of the level that has several last links: a lane takes its own one by one
#pragma unroll
      for (int i = 0; i < kNodes; ++i) {
        if ((levels[i / 4] >> (i % 4 * 8) & 0xffu) != (uint32_t)l) continue;
        if (from[i] & kSeveral) {
          several |= 1u << i;
          continue;
        }
        const int v = tid + i * kCostThreads;
        const double x = value[from[i]] + price[i];
        value[v] = x;
        near(c.cost + row, v) = x;
      }
      while (several != 0) {
        const int v = tid + __builtin_ctz(several) * kCostThreads;
        several &= several - 1;
        SmallRow<KS> r;
        r.load(c.in, 8 * v);
        const double x = cost_mean<KS>(c, of, r, last_links(r, level, l), v);
        value[v] = x;
        c.cost[row + v] = x;
      }
      lds_barrier();
    }
    __syncthreads();
  }
}

// The same with costs where they go, in memory, for more nodes than LDS has doubles for.
template <int KS>
__global__ void __launch_bounds__(kCostThreads) k_cost_scan_memory(CostView c) {
  extern __shared__ __align__(16) unsigned char cost_state[];
  unsigned char* const level = cost_state;
  const int N = c.N;
  for (int s = blockIdx.x; s < c.sources; s += gridDim.x) {
    const size_t row = (size_t)s * N;
    double* const value = c.cost + row;
    const double* const sigma = c.sigma + row;
    const auto of = [&](uint32_t u) { return make_double2(sigma[u], value[u]); };
    for (int v = threadIdx.x; v < N; v += kCostThreads) {
      const int d = c.dist[row + v];
      const int l = (unsigned)d <= (unsigned)c.depth ? d : kSmallUnseen;
      level[v] = (unsigned char)l;
      if (l == 0 || l == kSmallUnseen) value[v] = 0.0;
    }
    __syncthreads();
    for (int l = 1; l <= c.depth; ++l) {
      for (int v = threadIdx.x; v < N; v += kCostThreads) {
        if (level[v] != l) continue;
        SmallRow<KS> r;
        r.load(c.in, 8 * v);
        const uint32_t mask = last_links(r, level, l);
        if ((mask & (mask - 1)) == 0) {
          int place;
          uint32_t from;
          only_link(r, mask, place, from);
          value[v] = value[from] + (c.link_cost != nullptr ? near(c.prices, price_at(place, v, N)) : 1.0);
        } else {
          value[v] = cost_mean<KS>(c, of, r, mask, v);
        }
      }
      __syncthreads();
    }
  }
}

// Many sources of more nodes, a launch a level.  First a byte with its level and the places of its last links for every node, a
// workgroup per source with the level bytes in LDS; also the costs that need no link.
template <int KS>
__global__ void __launch_bounds__(kCostThreads) k_cost_marks(CostView c) {
  extern __shared__ __align__(16) unsigned char cost_state[];
  unsigned char* const level = cost_state;
  const int N = c.N;
  const size_t row = (size_t)blockIdx.x * N;
  for (int v = threadIdx.x; v < N; v += kCostThreads) {
    const int d = c.dist[row + v];
    const int l = (unsigned)d <= (unsigned)c.depth ? d : kSmallUnseen;
    level[v] = (unsigned char)l;
    c.levels[row + v] = (unsigned char)l;
    if (l == 0 || l == kSmallUnseen) c.cost[row + v] = 0.0;
    if (l == 0) c.pairs[row + v] = make_double2(c.sigma[row + v], 0.0);
  }
  __syncthreads();
  for (int v = threadIdx.x; v < N; v += kCostThreads) {
    SmallRow<KS> r;
    r.load(c.in, 8 * v);
    c.masks[row + v] = (uint16_t)last_links(r, level, level[v]);
  }
}

// Then the nodes of one level.  A workgroup has kCostLevelNodes of a source; workgroups go to the 8 XCDs in turn, and those of an
// XCD have the parts of its sources one after the other, so that the path counts and costs that they gather, 1 MB a source of
// 65536 nodes, stay in its L2; the two lie beside each other, one request for both.  1024 sources of 65536 nodes of degree 8: 4.0 ms, 5.8 by
// k_cost_scan_memory, which fetches twice as much past L2 (18 GB).  Bound by what L1 does not have: 275 of 579 million lookups go on to
// L2, and L1 stands still for it 55 % of the time (lookups alone would take a quarter, the 9.1 GB read and 2.8 written past L2 less than 3 ms).
template <int KS>
__global__ void __launch_bounds__(kCostLevelThreads) k_cost_level(CostView c, int l, int parts) {
  const int k = blockIdx.x / kXcd, s = k / parts * kXcd + blockIdx.x % kXcd;
  if (s >= c.sources) return;
  const size_t row = (size_t)s * c.N;
  double2* const pairs = c.pairs + row;
  const auto of = [&](uint32_t u) { return pairs[u]; };
  for (int i = 0; i < kCostLevelNodes / kCostLevelThreads; ++i) {
    const int v = k % parts * kCostLevelNodes + i * kCostLevelThreads + threadIdx.x;
    if (v >= c.N || c.levels[row + v] != l) continue;
    const uint32_t mask = c.masks[row + v];
    const double paths = c.sigma[row + v];
    SmallRow<KS> r;
    r.load(c.in, 8 * v);
    double x;
    if ((mask & (mask - 1)) == 0) {
      int place;
      uint32_t from;
      only_link(r, mask, place, from);
      x = pairs[from].y + (c.link_cost != nullptr ? near(c.prices, price_at(place, v, c.N)) : 1.0);
    } else {
      x = cost_mean<KS>(c, of, r, mask, v);
    }
    pairs[v] = make_double2(paths, x);
    c.cost[row + v] = x;
  }
}

// A workgroup per source, everything in memory, a level of all nodes at a time: topologies without a link table, deep
// ones and large ones.
static __global__ void __launch_bounds__(kCostThreads) k_cost_levels(CostView c) {
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
