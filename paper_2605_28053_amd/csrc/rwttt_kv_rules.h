// Rules of the paged cache's kernels as functions of numbers alone, for the
// device and for the host: C++ without HIP, so that they can be checked on any
// machine.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace rwttt {

// More LDS than this in a launch has to be asked for; a CU has 160 KB.
constexpr size_t kPlainLds = 64 * 1024;

// ---------------------------------------------------------------------------
// extend: what a step is refused for
// ---------------------------------------------------------------------------

enum class ExtendVerdict { ok, invalid, capacity };

// lengths_ok: every length in range.  The ring has room for the pages that come
// back beside all those it holds: pages taken and pages returned in one call are
// read and written at once, so the places must not meet.
constexpr ExtendVerdict extend_verdict(bool lengths_ok, int front, int count, int pages, long long taken,
                                       long long given, long long added, uint32_t cap) {
  if (!lengths_ok || front < 0 || front >= pages || count < 0 || count > pages) return ExtendVerdict::invalid;
  if (taken > count || added > cap) return ExtendVerdict::capacity;
  if (count + given > pages) return ExtendVerdict::invalid;
  return ExtendVerdict::ok;
}

// ---------------------------------------------------------------------------
// select: which scores are kept
// ---------------------------------------------------------------------------

// What the queries of a group, with a the largest magnitude, are multiplied by before
// they are rounded to 8 bits.  Queries so small that it is no fp32 number count as 0.
constexpr float query_unit(float a) {
  const float to = a > 0.f ? 1.f / a * 127.f : 0.f;
  return to < __builtin_inff() ? to : 0.f;
}

constexpr int kSelBits = 12, kSelBins = 1 << kSelBits;

constexpr int kSelThreads = 512, kSelWaves = kSelThreads / 64;

struct alignas(8) ScoredPage {
  uint32_t score, page;
};

// A block's LDS beside its scores (4 bytes a page, the launch's dynamic part).
template <int D> struct SelectLds {
  alignas(16) uint32_t hist[kSelBins];
  alignas(16) uint32_t digits[4][D / 4];   // U's low and high digit, V's low and high digit
  ScoredPage close[kSelThreads];
  uint32_t wave_least[kSelWaves], wave_most[kSelWaves], wave_sum[2][kSelWaves];
  float wave_max[kSelWaves];
  uint32_t pick[4];
};

// Scores of a table of max_pages pages, an even number of them.
constexpr int select_pitch(int max_pages) { return (max_pages + 1) & ~1; }
constexpr size_t select_lds(int max_pages) { return size_t(select_pitch(max_pages)) * sizeof(uint32_t); }
template <int D> constexpr bool select_asks_for_lds(int max_pages) {
  return select_lds(max_pages) + sizeof(SelectLds<D>) > kPlainLds;
}

// The state of a ranking of v = score - least, narrowed by the bin that the last
// kept one lies in.  Kept are all v > v0, and of those equal to v0 the first `want`.
// While bits below `top` are open, v0's are zero and `want` counts the bin's.
struct Rank {
  uint32_t v0;
  int want, top;
};

// want >= 1 of the values in [0, range].
constexpr Rank rank_begin(uint32_t range, int want) { return {0, want, range ? 32 - __builtin_clz(range) : 0}; }

constexpr int rank_bit(const Rank& r) { return r.top > kSelBits ? r.top - kSelBits : 0; }

// Whether v lies in the bin that is looked at, and its bin within.
constexpr bool rank_in(const Rank& r, uint32_t v) { return r.top == 32 || v >> r.top == r.v0 >> r.top; }
constexpr uint32_t rank_bin(const Rank& r, uint32_t v) { return (v >> rank_bit(r)) & (kSelBins - 1); }

// The last kept one lies in `bin`, which holds `count` values, with `above` in the
// bins over it.  A bin that is kept whole ends the ranking.
constexpr Rank rank_narrow(Rank r, uint32_t bin, int above, int count) {
  const int bit = rank_bit(r);
  r.v0 |= bin << bit;
  r.want -= above;
  r.top = bit;
  if (count == r.want) {
    r.top = 0;
    if (r.v0) {
      r.v0 -= 1;
      r.want = 0;
    }
  }
  return r;
}

// ---------------------------------------------------------------------------
// attend: the line of all rows' tiles, and where it is cut
// ---------------------------------------------------------------------------
//
// A row (an owner, kv head and sixteen queries) of t > 0 tiles has the cost t +
// kRowCost, and the rows' costs one after another are the line.  It is cut into
// equal parts, one a block.  The device knows the owners' lengths and cuts; the
// host launches as many blocks as the longest owners could have parts.

// A row's fixed cost in tiles: finding its pages, starting its loads and adding
// the waves' sums.  Counted in the line that is cut, it keeps a block from being
// dealt dozens of short rows against another's one long one: 32 owners of 1 to
// 40000 rows in e4m3 take 150 us without it, 115, 101, 88, 90 and 91 us with 2,
// 4, 8, 16 and 24 tiles.
constexpr int kRowCost = 8;
constexpr uint32_t row_cost(int tiles) { return uint32_t(tiles ? tiles + kRowCost : 0); }

// Part w of [0, total) cut into `parts` parts, the first ones one longer.
struct Cut {
  uint64_t per, rem;
  constexpr Cut(uint64_t total, int parts) : per(0), rem(0) {
    if (total >> 32) {                   // 64-bit division is a long routine
      per = total / parts;
      rem = total % parts;
    } else {
      per = uint32_t(total) / uint32_t(parts);
      rem = uint32_t(total) % uint32_t(parts);
    }
  }
  constexpr uint64_t begin(uint64_t w) const { return w * per + (w < rem ? w : rem); }
  constexpr int part_of(uint64_t u) const {
    const uint64_t head = rem * (per + 1);
    const uint64_t x = u < head ? u : u - head, by = u < head ? per + 1 : per;
    const uint64_t at = x >> 32 || by >> 32 ? x / by : uint32_t(x) / uint32_t(by);
    return int(u < head ? at : rem + at);
  }
};

// Smallest part of the line: a short row, or a few tiles of a long one.  One owner
// of 4224 rows takes 15.0, 13.5, 13.1 and 13.3 us with 4, 6, 8 and 12: smaller parts
// have more results to join.
constexpr int kPartCost = 8;
constexpr int parts_of(uint64_t total, int blocks) {
  return total >= uint64_t(blocks) * kPartCost ? blocks : int(uint32_t(total + kPartCost - 1) / kPartCost);
}

// Blocks of a launch for `rows` rows of at most `longest` keys each, in tiles of
// `tile`: the parts of the longest line there can be, so that no part is without one.
constexpr int attend_grid(uint64_t rows, int longest, int tile, int blocks) {
  return parts_of(rows * row_cost((longest + tile - 1) / tile), blocks);
}

// Whether the cache's rows are loaded with the non-temporal hint: where one step
// may read more than a quarter of the last-level cache's 256 MB over all layers.  The
// rest of a step (the owners' fast weights, the projections) then leaves nothing of
// them for the next one, and the hint keeps them from displacing what is there.  In
// us with / without the hint: 331 / 374 for 32 owners of 12000-20000 rows (2.2 GB),
// 31.3 / 33.2 for eight of 4200 (136 MB) where 270 MB of others are read in between,
// and 32.4 / 30.8 where only as much is; below, a step finds the last one's rows in
// the cache: 12.3 / 11.4 for one owner of 4224 (17 MB), 10.9 / 8.9 for eight of 300, 19.8
// / 17.1 for 32 of 400 (52 MB).
// The lengths are on the device, so the rule takes the most that the arguments
// allow: the pool, or what the listed owners can hold, list or have in the window.
// Short contexts in a large pool get the hint, and lose what the last figures say,
// if they are all that runs.  A choice on the device, by the lengths, would save
// them that, but with both loops in one kernel every call takes 0.4 to 0.6 us
// longer and the largest 337 instead of 332.
constexpr uint64_t kStreamBytes = uint64_t(64) << 20;
constexpr bool attend_streams(uint64_t n_pages, uint64_t owners, uint64_t max_pages, uint64_t keep, uint64_t window,
                              uint64_t page_rows, uint64_t page_bytes, uint64_t layers) {
  const uint64_t spanned = (window + 2 * page_rows - 2) / page_rows;    // pages that a window can touch
  uint64_t each = keep ? keep : window ? spanned : max_pages;
  each = each < max_pages ? each : max_pages;
  const uint64_t pages = owners * each < n_pages ? owners * each : n_pages;
  return pages * page_bytes * layers > kStreamBytes;
}

// A cut that falls in a short row, or near an end of a long one, moves to the
// row's end: joining costs more than the imbalance (64 owners of up to 300 rows 17.2
// -> 13.4 us; 24 tiles as the bound of a short row measure the same).
constexpr uint32_t kShortRow = kRowCost + 12, kRowHead = kRowCost + 3, kRowTail = 3;
static_assert(kShortRow > kRowHead + kRowTail, "a row that is split keeps a middle");
constexpr uint32_t snapped(uint32_t x, uint32_t cost) {
  if (cost <= kShortRow || x <= kRowHead) return 0;
  return x >= cost - kRowTail ? cost : x;
}

// The first and last of the parts that hold some of the row of this cost that
// begins at u0, by its cuts as they are snapped.
constexpr int first_part(const Cut& cut, uint64_t u0) { return cut.part_of(u0 + kRowHead); }
constexpr int last_part(const Cut& cut, uint64_t u0, uint32_t cost) { return cut.part_of(u0 + cost - kRowTail - 1); }

}  // namespace rwttt
