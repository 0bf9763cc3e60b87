// Prints the answers of the paged cache's rules, one line for each query line of stdin:
//   rank want close n s0 .. s(n-1)   -> the kept indices; bins of at most `close` scores are
//                                       ranked one by one
//   extend front count pages taken given added cap -> 0 ok, 1 invalid, 2 capacity, and for a step
//                                       that is ok the places of the ring both read and written
//   lds dim max_pages                -> bytes of LDS of a select's block, 1 if they are asked for
//   stream n_pages owners max_pages keep window page_rows page_bytes layers -> 1 if loaded with the hint
//   unit a                           -> query_unit's bits
//   cut blocks vh tile longest n l0 .. l(n-1) -> blocks launched, parts, parts of no block, tiles
//                                       that are not held by one launched part alone, rows whose
//                                       first and last part are not those that hold them
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <iostream>
#include <string>
#include <vector>

#include "rwttt_kv_rules.h"

using namespace rwttt;

static void rank(int want, int close, const std::vector<long long>& score) {
  std::vector<uint32_t> v;
  const long long least = *std::min_element(score.begin(), score.end());
  for (long long s : score) v.push_back(uint32_t(s - least));
  Rank r = rank_begin(*std::max_element(v.begin(), v.end()), want);
  while (r.top > 0) {
    std::vector<int> hist(kSelBins);
    for (uint32_t x : v)
      if (rank_in(r, x)) ++hist[rank_bin(r, x)];
    int above = 0, bin = kSelBins - 1;
    while (above + hist[bin] < r.want) above += hist[bin--];
    r = rank_narrow(r, uint32_t(bin), above, hist[bin]);
    if (r.top > 0 && hist[bin] <= close) {
      std::vector<uint32_t> in;
      for (uint32_t x : v)
        if (rank_in(r, x)) in.push_back(x);
      std::sort(in.rbegin(), in.rend());
      const uint32_t last = in[r.want - 1];
      r.want -= int(std::count_if(in.begin(), in.end(), [&](uint32_t x) { return x > last; }));
      r.v0 = last;
      r.top = 0;
    }
  }
  int equal = 0;
  for (size_t j = 0; j < v.size(); ++j)
    if (v[j] > r.v0 || (v[j] == r.v0 && equal++ < r.want)) std::printf("%zu ", j);
  std::printf("\n");
}

// attend's walk of the line of n owners' rows (vh each), the parts one after another.
static void cut_line(int blocks, int vh, int tile, int longest, const std::vector<int>& len) {
  const int n = int(len.size());
  std::vector<uint64_t> pre(n + 1);
  for (int i = 0; i < n; ++i) pre[i + 1] = pre[i] + row_cost((len[i] + tile - 1) / tile);
  const uint64_t total = pre[n] * vh;
  const int grid = attend_grid(uint64_t(n) * vh, longest, tile, blocks), parts = parts_of(total, blocks);
  std::vector<std::vector<int>> held(size_t(n) * vh);       // launched parts that hold each tile
  std::vector<std::vector<int>> by(size_t(n) * vh);         // parts that hold some of the row
  for (int r = 0; r < n * vh; ++r) held[r].resize((len[r / vh] + tile - 1) / tile);
  const Cut cut(total ? total : 1, parts ? parts : 1);
  auto begin = [&](int b) {
    const uint64_t u = cut.begin(b);
    if (u >= total) return total;
    int i = 0;
    while (pre[i + 1] * vh <= u) ++i;
    const uint32_t cost = uint32_t(pre[i + 1] - pre[i]), x = uint32_t(u - pre[i] * vh) % cost;
    return u + snapped(x, cost) - x;
  };
  for (int b = 0; b < std::min(grid, parts); ++b) {
    const uint64_t u = begin(b), end = begin(b + 1);
    for (int r = 0; r < n * vh; ++r) {
      const uint64_t u0 = pre[r / vh] * vh + (r % vh) * (pre[r / vh + 1] - pre[r / vh]);
      const uint64_t cost = pre[r / vh + 1] - pre[r / vh], x0 = std::max(u, u0), x1 = std::min(end, u0 + cost);
      if (x0 >= x1) continue;
      by[r].push_back(b);
      for (uint64_t t = std::max<int64_t>(0, int64_t(x0 - u0) - kRowCost); int64_t(t) < int64_t(x1 - u0) - kRowCost; ++t)
        ++held[r][t];
    }
  }
  int wrong = 0, joins = 0;
  for (int r = 0; r < n * vh; ++r) {
    for (int x : held[r]) wrong += x != 1;
    if (held[r].empty() || by[r].size() == 1) continue;
    const uint64_t u0 = pre[r / vh] * vh + (r % vh) * (pre[r / vh + 1] - pre[r / vh]);
    const int b0 = first_part(cut, u0), b1 = last_part(cut, u0, uint32_t(pre[r / vh + 1] - pre[r / vh]));
    joins += by[r].empty() || by[r].front() != b0 || by[r].back() != b1 || int(by[r].size()) != b1 - b0 + 1;
  }
  std::printf("%d %d %d %d %d\n", grid, parts, std::max(0, parts - grid), wrong, joins);
}

int main() {
  std::string what;
  while (std::cin >> what) {
    if (what == "rank") {
      int want, close, n;
      std::cin >> want >> close >> n;
      std::vector<long long> score(n);
      for (long long& s : score) std::cin >> s;
      rank(want, close, score);
    } else if (what == "extend") {
      int front, count, pages, taken, given, added, cap, meet = 0;
      std::cin >> front >> count >> pages >> taken >> given >> added >> cap;
      const ExtendVerdict v = extend_verdict(true, front, count, pages, taken, given, added, uint32_t(cap));
      if (v == ExtendVerdict::ok)
        for (int i = 0; i < given; ++i)
          for (int j = 0; j < taken; ++j) meet += (front + count + i) % pages == (front + j) % pages;
      std::printf("%d %d\n", int(v), meet);
    } else if (what == "lds") {
      int dim, pages;
      std::cin >> dim >> pages;
      const size_t fixed = dim == 64 ? sizeof(SelectLds<64>) : dim == 128 ? sizeof(SelectLds<128>) : sizeof(SelectLds<256>);
      const bool asks = dim == 64    ? select_asks_for_lds<64>(pages)
                        : dim == 128 ? select_asks_for_lds<128>(pages)
                                     : select_asks_for_lds<256>(pages);
      std::printf("%zu %d\n", fixed + select_lds(pages), asks);
    } else if (what == "stream") {
      uint64_t a[8];
      for (uint64_t& x : a) std::cin >> x;
      std::printf("%d\n", attend_streams(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]));
    } else if (what == "unit") {
      std::string text;
      std::cin >> text;
      const float unit = query_unit(std::strtof(text.c_str(), nullptr));
      uint32_t bits;
      std::memcpy(&bits, &unit, 4);
      std::printf("%u\n", bits);
    } else if (what == "cut") {
      int blocks, vh, tile, longest, n;
      std::cin >> blocks >> vh >> tile >> longest >> n;
      std::vector<int> len(n);
      for (int& l : len) std::cin >> l;
      cut_line(blocks, vh, tile, longest, len);
    }
  }
}
