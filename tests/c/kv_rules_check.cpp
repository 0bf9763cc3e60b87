// Prints the answers of the paged cache's rules, one line for each query line of stdin:
//   rank want close n s0 .. s(n-1)   -> the kept indices; bins of at most `close` scores are
//                                       ranked one by one
#include <algorithm>
#include <cstdio>
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

int main() {
  std::string what;
  while (std::cin >> what) {
    if (what == "rank") {
      int want, close, n;
      std::cin >> want >> close >> n;
      std::vector<long long> score(n);
      for (long long& s : score) std::cin >> s;
      rank(want, close, score);
    }
  }
}
