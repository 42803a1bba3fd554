// Device code of the dispatch functions: counts and demands of a router's choices, the balance loss and its gradient.
#pragma once

#include "a2a_dispatch_plan.h"
#include "a2a_kernels.h"

namespace a2a_dev {

// ---------------------------------------------------------------------------------------
// tokens and their sources
// ---------------------------------------------------------------------------------------

struct Routing {
  const void* choices;
  const int64_t* host_begin;
  const int32_t* expert_host;
  long long tokens, stride;
  int k, experts, sources;
};

// Entries of host_begin that are at most t: the source of token t is one less.  Of all lanes together, 64 parts of what
// is left at a time: three steps for up to 262143 sources.
__device__ __forceinline__ unsigned begun(const int64_t* __restrict__ begin, unsigned entries, long long t) {
  static_assert(kSearchParts == kWave);
  unsigned lo = 0, hi = entries;
  while (lo < hi) {
    const unsigned part = search_part(lo, hi), lane = (unsigned)lane_id();
    const unsigned at = search_behind(lo, hi, part, lane) - 1;
    const unsigned whole = (unsigned)__popcll(__ballot(begin[at] <= t && lo + lane * part < hi));
    // all of the parts before the first whose last entry is larger (of a last, shorter part too)
    if (lo + whole * part >= hi) return hi;
    lo += whole * part;
    hi = min(lo + part, hi) - 1;
  }
  return lo;
}

// ---------------------------------------------------------------------------------------
// counts and demands
// ---------------------------------------------------------------------------------------

// Cells are counted in LDS, by a workgroup that has them to itself (k_dispatch_tiles) or has some tokens of a source
// (k_dispatch_split).  Whole numbers: no order of additions matters.  What a choice counts for is a row: the expert
// (counts) or its host (demands).
struct Dispatch {
  Routing r;
  int rows, once;   // rows: experts or hosts
  int tile, tiles;  // rows of a workgroup
  int columns;      // sources of a workgroup
  long long per;    // tokens of a workgroup (k_dispatch_split)
  int32_t* counts;  // [sources][rows]
  double* demand;   // [rows][sources]
};

// Row of choice number i of the tokens from t0 on, and its token; -1: none.
template <typename Id, bool kDemand>
struct Choices {
  const Routing& r;
  const Id* at;
  int rows;
  bool once, dense;
  unsigned k;
  __device__ __forceinline__ Choices(const Dispatch& d, long long t0)
      : r(d.r), at((const Id*)d.r.choices + t0 * d.r.stride), rows(d.rows), once(d.once != 0), dense(d.r.stride == d.r.k), k(d.r.k) {}
  __device__ __forceinline__ Id raw(unsigned i) const { return dense ? at[i] : at[(long long)(i / k) * r.stride + i % k]; }
  __device__ __forceinline__ int row_of(Id e) const {
    if (e < 0 || e >= r.experts) return -1;
    if constexpr (!kDemand) return (int)e;
    const int h = r.expert_host ? r.expert_host[e] : (int)e;
    return (unsigned)h < (unsigned)rows ? h : -1;
  }
};

// f(i, row) for the choices i of n that a thread has and that count: of all, four of them asked for at a time; or of every
// token the first for each host, eight choices of a token at a time.
template <typename Id, bool kDemand, typename F>
__device__ __forceinline__ void each_row(const Choices<Id, kDemand>& c, unsigned n, F&& f) {
  if (kDemand && c.once) {
    constexpr unsigned kAhead = 8;
    const auto hosts = [&](unsigned i, unsigned left, int (&h)[kAhead]) {
      Id e[kAhead];
#pragma unroll
      for (unsigned q = 0; q < kAhead; ++q) e[q] = q < left ? c.raw(i + q) : (Id)-1;
#pragma unroll
      for (unsigned q = 0; q < kAhead; ++q) h[q] = c.row_of(e[q]);
    };
    for (unsigned t = threadIdx.x; t < n / c.k; t += blockDim.x)
      for (unsigned j = 0; j < c.k; j += kAhead) {
        int h[kAhead], before[kAhead];
        hosts(t * c.k + j, c.k - j, h);
#pragma unroll
        for (unsigned q = 1; q < kAhead; ++q)
#pragma unroll
          for (unsigned p = 0; p < q; ++p) h[q] = h[q] == h[p] ? -1 : h[q];
        for (unsigned i = 0; i < j; i += kAhead) {
          hosts(t * c.k + i, kAhead, before);
#pragma unroll
          for (unsigned q = 0; q < kAhead; ++q)
#pragma unroll
            for (unsigned p = 0; p < kAhead; ++p) h[q] = h[q] == before[p] ? -1 : h[q];
        }
#pragma unroll
        for (unsigned q = 0; q < kAhead; ++q)
          if (h[q] >= 0) f(t * c.k + j + q, h[q]);
      }
    return;
  }
  constexpr unsigned kAhead = 4;
  for (unsigned i0 = threadIdx.x; i0 < n; i0 += kAhead * blockDim.x) {
    Id e[kAhead];
#pragma unroll
    for (unsigned q = 0; q < kAhead; ++q) {
      const unsigned i = i0 + q * blockDim.x;
      e[q] = i < n ? c.raw(i) : (Id)-1;
    }
#pragma unroll
    for (unsigned q = 0; q < kAhead; ++q) {
      const int h = c.row_of(e[q]);
      if (h >= 0) f(i0 + q * blockDim.x, h);
    }
  }
}

static __global__ void __launch_bounds__(kBlock) k_fill(int32_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (size_t)gridDim.x * kBlock) p[i] = 0;
}

// host_begin as it may be used: within the tokens
__device__ __forceinline__ long long begin_of(const Routing& r, int s) {
  return min(max((long long)r.host_begin[s], 0ll), r.tokens);
}

// A band of `columns` sources and `tile` rows a workgroup, which reads these sources' tokens and writes the cells.  A cell has 16
// bits where the band has less than 65536 choices; where it has more, 32, and the rows go in two halves, each with a pass over
// the tokens.  Bound by the stores of large matrices: 4096 hosts, 524288 tokens of 8 choices, 134 MB, 31 us (4.3 TB/s); four passes over
// the tokens with cells of 32 bits took 106.
template <typename Id, bool kDemand>
__global__ void __launch_bounds__(kDispatchThreads) k_dispatch_tiles(Dispatch d) {
  extern __shared__ uint32_t cells[];  // demands: [rows][columns]
  __shared__ long long begin[kDispatchColumns + 1];
  __shared__ unsigned behind[kDispatchColumns];  // of the first choice of the band, behind the last one of a source
  const int T = blockDim.x;
  const int s0 = blockIdx.x / d.tiles * d.columns;
  const int columns = min(d.columns, d.r.sources - s0), band_rows = min(d.tile, d.rows - blockIdx.x % d.tiles * d.tile);
  if ((int)threadIdx.x <= columns) begin[threadIdx.x] = begin_of(d.r, s0 + threadIdx.x);
  __syncthreads();
  const long long t0 = begin[0];
  const unsigned k = d.r.k, n = begin[columns] > t0 ? (unsigned)(begin[columns] - t0) * k : 0;
  if ((int)threadIdx.x < kDispatchColumns)
    behind[threadIdx.x] = (int)threadIdx.x < columns ? (unsigned)(max(begin[threadIdx.x + 1], t0) - t0) * k : ~0u;
  const Choices<Id, kDemand> c(d, t0);
  const bool narrow = n < 65536u;
  const int part = narrow ? d.tile : (d.tile + 1) / 2;
  for (int done = 0; done < band_rows; done += part) {
    const int row0 = blockIdx.x % d.tiles * d.tile + done, rows = min(part, band_rows - done), size = rows * columns;
    const int words = narrow ? (size + 1) / 2 : size;
    for (int i = threadIdx.x; i < words; i += T) cells[i] = 0;
    __syncthreads();
    each_row<Id, kDemand>(c, n, [&](unsigned i, int h) {
      const unsigned row = (unsigned)(h - row0);
      if (row >= (unsigned)rows) return;
      unsigned s = 0;
      if constexpr (kDemand) {
#pragma unroll
        for (int half = kDispatchColumns / 2; half > 0; half /= 2) s += behind[s + half - 1] <= i ? half : 0;
      }
      const unsigned at = row * columns + s;
      narrow ? atomicAdd(&cells[at / 2], at & 1u ? 0x10000u : 1u) : atomicAdd(&cells[at], 1u);
    });
    __syncthreads();
    const auto cell = [&](int i) { return narrow ? cells[i / 2] >> (i & 1 ? 16 : 0) & 0xffffu : cells[i]; };
    if constexpr (kDemand) {
      if (columns == kDispatchColumns) {
        for (int i = threadIdx.x; i < size; i += T)
          d.demand[(size_t)(row0 + i / kDispatchColumns) * d.r.sources + s0 + i % kDispatchColumns] = (double)cell(i);
      } else {
        for (int i = threadIdx.x; i < size; i += T)
          d.demand[(size_t)(row0 + i / columns) * d.r.sources + s0 + i % columns] = (double)cell(i);
      }
    } else {
      for (int i = threadIdx.x; i < rows; i += T) d.counts[(size_t)s0 * d.rows + row0 + i] = (int32_t)cell(i);
    }
    __syncthreads();
  }
}

// `per` tokens a workgroup, their sources one after the other, into cells that are 0 before.  Bound by the loads: 68 MB of 64-bit
// choices of 1024 sources in 17 us (4.0 TB/s).
template <typename Id, bool kDemand>
__global__ void __launch_bounds__(kDispatchThreads) k_dispatch_split(Dispatch d) {
  extern __shared__ uint32_t cells[];  // [tile]
  const int T = blockDim.x;
  const int row0 = blockIdx.x % d.tiles * d.tile, rows = min(d.tile, d.rows - row0);
  long long t = (long long)(blockIdx.x / d.tiles) * d.per;
  const long long end = min(t + d.per, d.r.tokens);
  const auto add = [&](int s, int row, unsigned n) {
    if constexpr (kDemand)
      unsafeAtomicAdd(d.demand + (size_t)(row0 + row) * d.r.sources + s, (double)n);
    else
      atomicAdd(d.counts + (size_t)s * d.rows + row0 + row, (int)n);
  };
  while (t < end) {
    const int n = (int)begun(d.r.host_begin, d.r.sources + 1u, t);
    if (n > d.r.sources) break;
    const long long next = max(min(end, (long long)d.r.host_begin[n]), t + 1);
    if (n > 0) {
      const unsigned choices = (unsigned)(next - t) * d.r.k;
      const Choices<Id, kDemand> c(d, t);
      if (choices < (unsigned)rows / 4) {  // fewer than there are cells to look through
        each_row<Id, kDemand>(c, choices, [&](unsigned, int h) {
          const unsigned row = (unsigned)(h - row0);
          if (row < (unsigned)rows) add(n - 1, (int)row, 1);
        });
      } else {
        for (int i = threadIdx.x; i < rows; i += T) cells[i] = 0;
        __syncthreads();
        each_row<Id, kDemand>(c, choices, [&](unsigned, int h) {
          const unsigned row = (unsigned)(h - row0);
          if (row < (unsigned)rows) atomicAdd(&cells[row], 1u);
        });
        __syncthreads();
        for (int i = threadIdx.x; i < rows; i += T)
          if (cells[i] != 0) add(n - 1, i, cells[i]);
        __syncthreads();
      }
    }
    t = next;
  }
}

// ---------------------------------------------------------------------------------------
// balance loss
// ---------------------------------------------------------------------------------------
//
// Bound by memory: of 1048576 rows of 256 numbers in bfloat16 the forward pass reads 604 MB in 168 us and the gradient reads and
// writes 1074 MB in 202, in turn (5.3 TB/s; the copy of 1 GiB 4.8 to 5.1).  With 250 vector instructions for four rows the forward
// pass would take 130 us without memory, so they are kept few: sums across lanes by DPP, rows by pointers that are stepped.
//
// A row of logits lies in kLanes lanes, kValues numbers in each, and a wave has 64 / kLanes rows at a time: maximum and sum
// are taken in the lane first and between the lanes of a row then.  A lane keeps the sums of its experts' probabilities
// for as long as the source stays the same; what the waves of a workgroup have for it is added up once a piece.

struct Balance {
  Routing r;
  const void* logits;
  long long logits_stride, per;
  const double* cost;
  int hosts;
  // places of pieces (a2a_dispatch_plan.h)
  float* sums;
  int32_t* counts;
  int32_t* rows;
  // the call's
  double* terms;      // [workgroups of k_balance_sources][2]
  int across, wide_choices;
  float* out_loss;
  int32_t* out_counts;
  float* out_sums;
  int32_t* out_rows;
  // gradient
  const int32_t* in_counts;
  const int32_t* in_rows;
  const float* upstream;
  void* grad;
  long long grad_stride;
};

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kCtrl, 0xf, 0xf, true));
}

// f over the kLanes lanes of a row, in all of them.  Lanes of a quad, then of halves and wholes of 16 (mirrored: the quads
// agree by then), then across.
template <int kLanes, typename F>
__device__ __forceinline__ float over_lanes(float x, F f) {
  if constexpr (kLanes > 1) x = f(x, dpp<0xb1>(x));
  if constexpr (kLanes > 2) x = f(x, dpp<0x4e>(x));
  if constexpr (kLanes > 4) x = f(x, dpp<0x141>(x));
  if constexpr (kLanes > 8) x = f(x, dpp<0x140>(x));
  if constexpr (kLanes > 16) x = f(x, __shfl_xor(x, 16, kWave));
  if constexpr (kLanes > 32) x = f(x, __shfl_xor(x, 32, kWave));
  return x;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__bf16 x) { return (float)x; }
__device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }

// The numbers of a row that a lane has: pieces of 16 bytes (kWide: rows begin at multiples of 16 bytes and end at one), or one
// number at a time, neighbours in neighbouring lanes.  Requests for a row have no conditions, so that the next one's can be
// counted while this one's are waited for: a lane with a place past the row's end asks for the row's first piece and has
// -infinity in its place.
template <typename T, bool kWide, int kLanes, int kValues>
struct Row {
  static constexpr int kPiece = kWide ? 16 / (int)sizeof(T) : 1;
  static constexpr int kPieces = kValues / kPiece;
  typedef T Piece __attribute__((ext_vector_type(kPiece)));
  Piece p[kPieces];

  static __device__ __forceinline__ int expert(int lane, int i) {  // of a lane's number i
    return (i / kPiece * kLanes + lane) * kPiece + i % kPiece;
  }
  __device__ __forceinline__ void load(const T* row, int lane, int experts) {
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      const int e = expert(lane, q * kPiece);
      p[q] = *reinterpret_cast<const Piece*>(row + (e < experts ? e : 0));
    }
  }
  __device__ __forceinline__ void cut(int lane, int experts) {
#pragma unroll
    for (int q = 0; q < kPieces; ++q) p[q] = expert(lane, q * kPiece) < experts ? p[q] : (Piece)(T)-INFINITY;
  }
  __device__ __forceinline__ void store(T* __restrict__ row, int lane, int experts) const {
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      const int e = expert(lane, q * kPiece);
      if (e < experts) *reinterpret_cast<Piece*>(row + e) = p[q];
    }
  }
  __device__ __forceinline__ float get(int i) const { return to_float(p[i / kPiece][i % kPiece]); }
  __device__ __forceinline__ void set(int i, float x) { p[i / kPiece][i % kPiece] = (T)x; }

  // x[i] = exp(z_i - maximum); returns their sum over the row, 0 for a row of -infinity alone.  (exp2(z log2(e) - maximum log2(e))
  // by one multiply-add would be off by the rounding of the second product, which for a row of a mask's lowest values is
  // past any exponent.)
  __device__ __forceinline__ float exponentials(float (&x)[kValues]) const {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kValues; ++i) top = fmaxf(top, get(i));
    top = over_lanes<kLanes>(top, [](float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); });  // the larger one
    constexpr float kLog2e = 1.44269504088896340736f;
    top = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      x[i] = __builtin_amdgcn_exp2f((get(i) - top) * kLog2e);
      sum += x[i];
    }
    return over_lanes<kLanes>(sum, [](float a, float b) { return a + b; });
  }
};

// The pieces of workgroup b, in order: f(source, first token, token behind the last).  The end of the source after comes with
// the end of each, so that only sources behind empty ones are looked for.
template <typename F>
__device__ __forceinline__ void for_pieces(const Routing& r, long long per, F&& f) {
  long long t = (long long)blockIdx.x * per;
  const long long end = min(t + per, r.tokens);
  if (t >= end) return;
  const unsigned sources = r.sources;
  unsigned n = begun(r.host_begin, sources + 1, t);  // entries that are at most t
  while (n <= sources) {                             // not behind the last source's tokens
    const long long stop = r.host_begin[n], after = r.host_begin[min(n + 1, sources)];
    const long long next = max(min(end, stop), t + 1);
    if (n > 0) f((int)(n - 1), t, next);
    t = next;
    if (t >= end) break;
    n = stop == t && after > t ? n + 1 : begun(r.host_begin, sources + 1, t);
  }
}

// Sum over the rows that a wave has at a time, in the first row's lanes.
template <int kLanes>
__device__ __forceinline__ float over_rows(float x) {
  if constexpr (kLanes <= 1) x += dpp<0x121>(x);  // rotations within 16 lanes
  if constexpr (kLanes <= 2) x += dpp<0x122>(x);
  if constexpr (kLanes <= 4) x += dpp<0x124>(x);
  if constexpr (kLanes <= 8) x += dpp<0x128>(x);
  if constexpr (kLanes <= 16) x += __shfl_xor(x, 16, kWave);
  if constexpr (kLanes <= 32) x += __shfl_xor(x, 32, kWave);
  return x;
}

// Whether a lane asks for its next row before it works on the one it has: not where their registers are too many.
constexpr bool row_ahead(int values) { return values <= 40; }

template <typename T, bool kWide, int kLanes, int kValues>
__global__ void __launch_bounds__(kBalanceThreads) k_balance_rows(Balance b) {
  using R = Row<T, kWide, kLanes, kValues>;
  constexpr int kWaves = kBalanceThreads / kWave, kRows = kWave / kLanes, kStep = kWaves * kRows;
  extern __shared__ float lds[];  // [kWaves][experts] sums, int [experts] counts, int [kWaves] rows
  const int X = b.r.experts, k = b.r.k;
  int* const counts = (int*)(lds + kWaves * X);
  int* const rows = counts + X;
  const int wave = threadIdx.x / kWave, lane = lane_id() % kLanes, slot = lane_id() / kLanes;
  // the words of a choice as they come, and the expert that they say
  const int words = b.wide_choices ? 2 : 1;
  const auto choice = [&](const int32_t* p) { return make_int2(p[0], p[words - 1]); };
  const auto expert_of = [&](int2 e) { return (words == 1 || e.y == 0) && (unsigned)e.x < (unsigned)X ? e.x : -1; };
  const long long row_step = b.logits_stride * kStep, choice_step = b.r.stride * words * kStep;
  for_pieces(b.r, b.per, [&](int s, long long t0, long long t1) {
    R rows_of[2];  // a row is asked for while the one before is worked on; after the last one that again
    int2 marks[2];
    const int first = wave * kRows + slot, n = (int)(t1 - t0);
    int left = n - first;
    const T* at = (const T*)b.logits + (t0 + min(first, n - 1)) * b.logits_stride;
    const int32_t* choices = (const int32_t*)b.r.choices + (t0 + min(first, n - 1)) * b.r.stride * words;
    const auto fetch = [&](int i) {
      rows_of[i].load(at, lane, X);
      marks[i] = choice(choices + min(lane, k - 1) * words);
    };
    const auto next = [&] {
      at += left > kStep ? row_step : 0;
      choices += left > kStep ? choice_step : 0;
    };
    fetch(0);
    for (int i = threadIdx.x; i < X; i += kBalanceThreads) counts[i] = 0;
    __syncthreads();
    float acc[kValues] = {};
    int mine = 0;
    const auto work = [&](int i, const int32_t* of_row) {
      float x[kValues];
      rows_of[i].cut(lane, X);
      const float sum = rows_of[i].exponentials(x);
      const float inv = sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum);
#pragma unroll
      for (int j = 0; j < kValues; ++j) acc[j] = __builtin_fmaf(x[j], inv, acc[j]);
      if (sum == 0.0f) return;
      mine += lane == 0;
      const int e = lane < k ? expert_of(marks[i]) : -1;
      if (e >= 0) atomicAdd(&counts[e], 1);
      for (int j = lane + kLanes; j < k; j += kLanes) {
        const int more = expert_of(choice(of_row + j * words));
        if (more >= 0) atomicAdd(&counts[more], 1);
      }
    };
    while (left > 0) {
      const int32_t* const of_row = choices;
      next();
      if constexpr (row_ahead(kValues)) {
        fetch(1);
        work(0, of_row);
        left -= kStep;
        if (left <= 0) break;
        const int32_t* const of_next = choices;
        next();
        fetch(0);
        work(1, of_next);
      } else {
        work(0, of_row);
        fetch(0);
      }
      left -= kStep;
    }
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const float sum = over_rows<kLanes>(acc[i]);
      const int at = R::expert(lane, i);
      if (slot == 0 && at < X) lds[wave * X + at] = sum;
    }
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) mine += __shfl_xor(mine, m, kWave);
    if (lane_id() == 0) rows[wave] = mine;
    __syncthreads();
    const size_t place = (size_t)blockIdx.x + s;
    for (int i = threadIdx.x; i < X; i += kBalanceThreads) {
      float sum = lds[i];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) sum += lds[w * X + i];
      b.sums[place * X + i] = sum;
      b.counts[place * X + i] = counts[i];
    }
    if (threadIdx.x == 0) {
      int n = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) n += rows[w];
      b.rows[place] = n;
    }
    __syncthreads();
  });
}

__device__ __forceinline__ double weight_of(const Balance& b, int s, int e) {
  if (!b.cost) return 1.0;
  const int h = b.r.expert_host ? b.r.expert_host[e] : e;
  return h >= 0 && h < b.hosts ? b.cost[(size_t)s * b.hosts + h] : 0.0;
}

// Sum over the workgroup, in thread 0, in a fixed order.
__device__ __forceinline__ double block_sum(double x, double* lds) {
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) x += __shfl_xor(x, m, kWave);
  if (lane_id() == 0) lds[threadIdx.x / kWave] = x;
  __syncthreads();
  double sum = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < (int)blockDim.x / kWave; ++w) sum += lds[w];
  __syncthreads();
  return sum;
}

// A source's pieces added up, `across` of them at a time beside each other, for kBalanceThreads / across experts; where one
// at a time is enough (across 1) the cells of several sources beside each other: an item.  Double precision from here on.  A
// workgroup has every gridDim.x-th item and leaves the sum of their terms.  All in an order that the sizes alone decide.
static __global__ void __launch_bounds__(kBalanceThreads) k_balance_sources(Balance b) {
  __shared__ double lds[kBalanceThreads], waves[kBalanceThreads / kWave];
  __shared__ int lds_counts[kBalanceThreads], lds_rows[kBalanceThreads];
  const int X = b.r.experts, across = b.across, experts = kBalanceThreads / across, parts = (X + experts - 1) / experts;
  const int i = threadIdx.x % experts, lane = threadIdx.x / experts;
  const long long cells = (long long)b.r.sources * X;
  const long long items = across > 1 ? (long long)b.r.sources * parts : (cells + kBalanceThreads - 1) / kBalanceThreads;
  double terms = 0.0, all_rows = 0.0;
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    int s = (int)(item / parts), e = (int)(item % parts) * experts + i;
    if (across == 1) {
      const long long cell = min(item * kBalanceThreads + threadIdx.x, cells - 1);
      s = (int)(cell / X);
      e = item * kBalanceThreads + threadIdx.x < cells ? (int)(cell % X) : X;
    }
    const long long first = begin_of(b.r, s), behind = begin_of(b.r, s + 1);
    const long long g0 = first / b.per, g1 = behind > first ? (behind - 1) / b.per : g0 - 1;
    double sum = 0.0;
    int count = 0, rows = 0;
#pragma unroll 8
    for (long long g = g0 + lane; g <= g1; g += across) {
      rows += b.rows[g + s];
      if (e < X) {
        sum += b.sums[(g + s) * X + e];
        count += b.counts[(g + s) * X + e];
      }
    }
    if (across > 1) {
      lds[threadIdx.x] = sum;
      lds_counts[threadIdx.x] = count;
      lds_rows[threadIdx.x] = rows;
      __syncthreads();
      for (int half = across / 2; half > 0; half /= 2) {
        if (lane < half) {
          sum += lds[threadIdx.x + half * experts];
          count += lds_counts[threadIdx.x + half * experts];
          rows += lds_rows[threadIdx.x + half * experts];
          lds[threadIdx.x] = sum;
          lds_counts[threadIdx.x] = count;
          lds_rows[threadIdx.x] = rows;
        }
        __syncthreads();
      }
    }
    if (lane == 0 && e < X) {
      b.out_sums[(size_t)s * X + e] = (float)sum;
      b.out_counts[(size_t)s * X + e] = count;
      if (rows > 0) terms += weight_of(b, s, e) * count * sum / rows;
      if (e == 0) {
        b.out_rows[s] = rows;
        all_rows += rows;
      }
    }
  }
  terms = block_sum(terms, waves);
  all_rows = block_sum(all_rows, waves);
  if (threadIdx.x == 0) {
    b.terms[2 * blockIdx.x] = terms;
    b.terms[2 * blockIdx.x + 1] = all_rows;
  }
}

// The loss from those sums.  (The last workgroup of k_balance_sources to come could add them up, but a release at the scope of
// the device by every workgroup, with what it has written still in the caches, made that kernel 50 us for 1024 sources of 256
// experts, where it takes 10 without.)
static __global__ void __launch_bounds__(kBalanceThreads) k_balance_loss(Balance b, int groups) {
  __shared__ double waves[kBalanceThreads / kWave];
  double sum = 0.0, rows = 0.0;
  for (int g = threadIdx.x; g < groups; g += kBalanceThreads) {
    sum += b.terms[2 * g];
    rows += b.terms[2 * g + 1];
  }
  sum = block_sum(sum, waves);
  rows = block_sum(rows, waves);
  if (threadIdx.x == 0) b.out_loss[0] = rows > 0.0 ? (float)(sum * b.r.experts / (b.r.k * rows)) : 0.0f;
}

template <typename T, bool kWide, int kLanes, int kValues>
__global__ void __launch_bounds__(kBalanceThreads) k_balance_grad(Balance b) {
  using R = Row<T, kWide, kLanes, kValues>;
  constexpr int kWaves = kBalanceThreads / kWave, kRows = kWave / kLanes, kStep = kWaves * kRows;
  extern __shared__ double lds64[];  // [kWaves] doubles, float [experts]
  float* const coef = (float*)(lds64 + kWaves + 1);
  const int X = b.r.experts;
  const int wave = threadIdx.x / kWave, lane = lane_id() % kLanes, slot = lane_id() / kLanes;
  double n = 0.0;
  for (unsigned s = threadIdx.x; s < (unsigned)b.r.sources; s += kBalanceThreads) n += b.in_rows[s];
  n = block_sum(n, lds64);
  if (threadIdx.x == 0) lds64[kWaves] = n > 0.0 ? (b.upstream ? (double)b.upstream[0] : 1.0) * X / (b.r.k * n) : 0.0;
  __syncthreads();
  const double scale = lds64[kWaves];
  const long long row_step = b.logits_stride * kStep, grad_step = b.grad_stride * kStep;
  for_pieces(b.r, b.per, [&](int s, long long t0, long long t1) {
    R rows_of[2];
    const int first = wave * kRows + slot, n = (int)(t1 - t0);
    int left = n - first;
    const T* at = (const T*)b.logits + (t0 + min(first, n - 1)) * b.logits_stride;
    T* to = (T*)b.grad + (t0 + min(first, n - 1)) * b.grad_stride;
    const auto next = [&] { at += left > kStep ? row_step : 0; };
    rows_of[0].load(at, lane, X);
    const double of_source = scale / max(b.in_rows[s], 1);
    for (int e = threadIdx.x; e < X; e += kBalanceThreads)
      coef[e] = (float)(of_source * weight_of(b, s, e) * b.in_counts[(size_t)s * X + e]);
    __syncthreads();
    float c[kValues];
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const int e = R::expert(lane, i);
      c[i] = e < X ? coef[e] : 0.0f;
    }
    const auto work = [&](R& row) {
      float x[kValues];
      row.cut(lane, X);
      const float sum = row.exponentials(x);
      float dot = 0.0f;
#pragma unroll
      for (int i = 0; i < kValues; ++i) dot = __builtin_fmaf(x[i], c[i], dot);
      dot = over_lanes<kLanes>(dot, [](float a, float b) { return a + b; });
      // 0 for no token also where the coefficients are no finite numbers.  (A choice a number: 131072 x 2048 266 us, 250 without; up to 512
      // experts nothing that can be measured.  A branch a wave is no better, a loop of its own for such coefficients slower below.)
      const bool token = sum != 0.0f;
      const float inv = token ? __builtin_amdgcn_rcpf(sum) : 0.0f;
      dot *= inv;
      R z;
#pragma unroll
      for (int i = 0; i < kValues; ++i) z.set(i, token ? x[i] * inv * (c[i] - dot) : 0.0f);
      z.store(to, lane, X);
      to += grad_step;
      left -= kStep;
    };
    while (left > 0) {
      next();
      if constexpr (row_ahead(kValues)) {
        rows_of[1].load(at, lane, X);
        work(rows_of[0]);
        if (left <= 0) break;
        next();
        rows_of[0].load(at, lane, X);
        work(rows_of[1]);
      } else {
        work(rows_of[0]);
        rows_of[0].load(at, lane, X);
      }
    }
    __syncthreads();
  });
}

}  // namespace a2a_dev
