// What the dispatch functions accept and how their calls are cut up: plain host arithmetic, no HIP, so that it can be
// checked over its whole range without a device.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "a2a_topo.h"

namespace a2a_dev {

constexpr int kMostChoices = 64;

inline size_t type_bytes(int type) {
  switch (type) {
    case A2A_F32: case A2A_I32: return 4;
    case A2A_BF16: case A2A_F16: return 2;
    case A2A_I64: return 8;
    default: return 0;
  }
}

inline bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// rows x stride numbers of `bytes` each stay within an address space
inline bool spans(int64_t rows, int64_t stride, size_t bytes) {
  return stride <= 0 || rows <= (int64_t)((uint64_t)INT64_MAX / bytes) / stride;
}

// Arguments that all dispatch functions have.  choices: whether they are read.
inline int check_routing(int32_t src_count, const a2a_routing* r, bool choices) {
  if (src_count < 0 || !r || r->tokens < 0 || r->experts < 1 || r->reserved != 0) return A2A_ERR_INVALID_ARG;
  if (r->choices_per_token < 1 || r->choices_per_token > kMostChoices) return A2A_ERR_INVALID_ARG;
  if (r->tokens > (int64_t)INT32_MAX / r->choices_per_token) return A2A_ERR_NOT_IMPLEMENTED;  // counts are 32 bits
  if (src_count > 0 && (!r->host_begin || !aligned_to(r->host_begin, 8))) return A2A_ERR_INVALID_ARG;
  if (!aligned_to(r->expert_host, 4)) return A2A_ERR_INVALID_ARG;
  if (!choices) return A2A_OK;
  if (r->choices_type != A2A_I32 && r->choices_type != A2A_I64) return A2A_ERR_INVALID_ARG;
  if (r->choices_stride < r->choices_per_token || !spans(r->tokens, r->choices_stride, 8)) return A2A_ERR_INVALID_ARG;
  if (src_count > 0 && r->tokens > 0 && (!r->choices || !aligned_to(r->choices, type_bytes(r->choices_type)))) return A2A_ERR_INVALID_ARG;
  return A2A_OK;
}

// A matrix of logits (or of their gradients) for the routing's tokens.
inline int check_logits(const a2a_routing* r, const void* logits, int type, int64_t stride) {
  if (type != A2A_F32 && type != A2A_BF16 && type != A2A_F16) return A2A_ERR_INVALID_ARG;
  if (r->experts > A2A_MOST_EXPERTS) return A2A_ERR_NOT_IMPLEMENTED;
  if (stride < r->experts || !spans(r->tokens, stride, 4)) return A2A_ERR_INVALID_ARG;
  if (r->tokens > 0 && (!logits || !aligned_to(logits, type_bytes(type)))) return A2A_ERR_INVALID_ARG;
  return A2A_OK;
}

// Counts and demands.  A workgroup has a band of sources to itself, reads their tokens and writes their cells once; sources with
// many tokens are split over workgroups that add to cells set to 0 before.  The first reads and writes everything once, but a source with
// most of the tokens is one workgroup's; the second is even, but adds a piece's cells one by one, in a second launch.  So few bands are
// split where they have more than 16384 choices each, by the mean, which is all that the host knows.  How long bands take, the largest source
// decides (us of a call by bands, split; 64 hosts, k = 4: 65536 tokens, even 8.8, 11.7, the largest source 4 times the mean 10.1, 11.9;
// 131072 even 8.9, 11.6, 4 times 16.7, 11.7; 262143 even 10.3, 11.8, 4 times, more than cells of 16 bits count, 55.9, 11.7; 81 hosts, 20011 x
// 6, once, 4 times 9.1, 17.5).  And counts are split where a piece has four times as many choices as cells (1048576 x 8 of 1024 sources, the
// largest 8 times the mean, 256 experts: 44 us by bands, 18.5 split).
constexpr int kDispatchThreads = 1024;
constexpr int kDispatchColumns = 16;    // sources of a band at the most: 128 bytes of a row of demands
constexpr int kDispatchCells = 65536;   // cells of 16 bits: 128 KB of LDS
constexpr int64_t kLaunchThreads = 0xffffffffll;  // of a launch, at the most
struct DispatchCut {
  bool split = false;
  int columns = 1, tile = 1, tiles = 1, threads = 256;
  int64_t per = 0, groups = 0;  // tokens of a workgroup that splits; workgroups of a launch
  int64_t sources = 0;          // of a launch: all of them, but for counts of very many
  size_t lds = 0;
};
inline DispatchCut dispatch_cut(int64_t sources, int64_t tokens, int64_t choices_per_token, int64_t rows, bool demand) {
  DispatchCut c;
  const int64_t choices = tokens * choices_per_token;
  // As many sources a band as leave 256 bands, or 128 where a row of demands does not end with a line of 64 bytes: bands then share
  // lines, the more the narrower they are (us with 256 and 128: 4095 hosts, 524288 x 8 choices 51.7, 40.8, 3249 hosts, 2130 x 7 36.1,
  // 31.2; 2048 hosts, 100000 x 8 10.1, 13.4, 1024 hosts, 4000 x 2 7.5, 8.7).
  const int64_t each = sources % 8 == 0 ? 512 : 256;
  while (demand && c.columns < kDispatchColumns && sources >= each * c.columns) c.columns *= 2;
  const int64_t bands = (sources + c.columns - 1) / c.columns;
  // pieces of the split form, with a pass over the rows' cells each
  const int64_t per = std::max<int64_t>((tokens + 1023) / 1024, (1024 + choices_per_token - 1) / choices_per_token);
  const int64_t pieces = (tokens + per - 1) / per + sources;
  c.split = bands < 256 ? choices / bands > 16384 : !demand && choices / pieces > 4 * rows;
  c.sources = sources;
  if (c.split) {
    c.columns = 1;
    c.tile = (int)std::min<int64_t>(rows, kDispatchCells / 4);
    c.tiles = (int)((rows + c.tile - 1) / c.tile);
    const int64_t most = kLaunchThreads / c.threads / c.tiles;  // pieces of a launch
    c.per = std::max(per, (tokens + most - 1) / most);
    c.groups = (tokens + c.per - 1) / c.per * c.tiles;
    c.lds = (size_t)c.tile * 4;
  } else {
    c.tile = (int)std::min<int64_t>(rows, kDispatchCells / c.columns);
    c.tiles = (int)((rows + c.tile - 1) / c.tile);
    if (!demand) c.sources = std::min(sources, kLaunchThreads / c.threads / c.tiles);  // (demands of as many do not fit the memory)
    c.groups = (c.sources + c.columns - 1) / c.columns * c.tiles;
    c.lds = ((size_t)(c.tile + 1) / 2 * c.columns + 1) * 4;  // of 16 bits each, or of 32 for half of the rows
    if (demand && choices / bands > 1024) c.threads = kDispatchThreads;
  }
  return c;
}

// The source that a token belongs to is searched for by a wave, 64 parts of what is left, [lo, hi), at a time.  Unsigned: there may be 2^31
// entries, and the place behind the last part is up to 63 further.
constexpr unsigned kSearchParts = 64;
constexpr unsigned search_part(unsigned lo, unsigned hi) { return (hi - lo + kSearchParts - 1) / kSearchParts; }
constexpr unsigned search_behind(unsigned lo, unsigned hi, unsigned part, unsigned n) {  // the n-th part's end
  return lo + (n + 1) * part < hi ? lo + (n + 1) * part : hi;
}

// Passes over logits: a workgroup has `per` consecutive tokens, of as many sources as they belong to.  The tokens of
// workgroup b that belong to source s are its piece (b, s).  Pieces follow each other, and from one to the next b or s
// grows, so b + s numbers them: the sums of a piece have place b + s of the workspace, and those of source s are the
// places b + s of the workgroups b that its tokens fall into.
constexpr int kBalanceThreads = 256;
struct BalanceCut {
  int64_t per = 0;     // tokens a workgroup
  int64_t groups = 0;  // workgroups
};
// As many workgroups as run at once (1536), but parts of 256 tokens where there would be less in them: what a workgroup spends on
// its first row and on each piece's sums (131071 x 160: parts of 64 tokens 18.8 us for 8 lanes a row, of 256 15.2, and a third of the pieces to add up).
inline BalanceCut balance_cut(int64_t tokens) {
  BalanceCut c;
  c.per = std::max<int64_t>({16, (tokens + 1535) / 1536, std::min<int64_t>(256, (tokens + 511) / 512)});
  c.groups = (tokens + c.per - 1) / c.per;
  return c;
}

// f(a row's shape) for `experts` numbers, in pieces of 16 bytes (wide) or single numbers: few lanes have few steps across lanes, but
// 8 of them or more read whole lines (160 numbers: 4 lanes of 40 23.5 us for 131071 rows, 8 of 24 18.8), and places that
// a row leaves empty cost as much as the others (16 lanes of 16 for the 160: 19.8).
template <bool kWide_, int kLanes_, int kValues_>
struct RowShape {
  static constexpr bool kWide = kWide_;
  static constexpr int kLanes = kLanes_, kValues = kValues_;
};
template <typename F>
void by_row(int experts, bool wide, F&& f) {
  if (!wide) {
    if (experts <= 128) return f(RowShape<false, 16, 8>{});
    if (experts <= 512) return f(RowShape<false, 16, 32>{});
    return f(RowShape<false, 64, 64>{});
  }
  if (experts <= 8) return f(RowShape<true, 1, 8>{});
  if (experts <= 16) return f(RowShape<true, 2, 8>{});
  if (experts <= 32) return f(RowShape<true, 4, 8>{});
  if (experts <= 64) return f(RowShape<true, 8, 8>{});
  if (experts <= 128) return f(RowShape<true, 16, 8>{});
  if (experts <= 192) return f(RowShape<true, 8, 24>{});
  if (experts <= 256) return f(RowShape<true, 16, 16>{});
  if (experts <= 320) return f(RowShape<true, 8, 40>{});
  if (experts <= 384) return f(RowShape<true, 16, 24>{});
  if (experts <= 512) return f(RowShape<true, 16, 32>{});
  if (experts <= 640) return f(RowShape<true, 16, 40>{});
  if (experts <= 1024) return f(RowShape<true, 16, 64>{});
  f(RowShape<true, 64, 64>{});
}

// Sums over a source's pieces: about four of them for a thread.
constexpr int kSourceGroups = 1024;  // workgroups at the most
struct SourceCut {
  int across = 1;
  int groups = 1;
};
inline SourceCut source_cut(int64_t sources, int64_t tokens, int64_t experts) {
  SourceCut c;
  const int64_t pieces = sources > 0 ? balance_cut(tokens).groups / sources + 1 : 1;
  while (c.across < 64 && pieces > 4 * c.across) c.across *= 2;
  const int64_t each = kBalanceThreads / c.across;
  const int64_t items = c.across > 1 ? sources * ((experts + each - 1) / each) : (sources * experts + each - 1) / each;
  c.groups = (int)std::max<int64_t>(1, std::min<int64_t>(kSourceGroups, items));
  return c;
}
struct BalanceLayout {
  size_t sums = 0, counts = 0, rows = 0, terms = 0, total = 0;
};
inline BalanceLayout balance_layout(int64_t src_count, int64_t tokens, int64_t experts) {
  const int64_t places = balance_cut(tokens).groups + src_count;
  BalanceLayout l;
  size_t off = 0;
  const auto part = [&off](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  l.sums = part((size_t)places * experts * 4);
  l.counts = part((size_t)places * experts * 4);
  l.rows = part((size_t)places * 4);
  l.terms = part((size_t)source_cut(src_count, tokens, experts).groups * 16);
  l.total = off;
  return l;
}

}  // namespace a2a_dev
