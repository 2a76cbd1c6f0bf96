// A run's search for its `keep` largest scores on the host: the search of k_select_search.h with the wavefront's 64 lanes as
// loops, KPL scores to a lane.  Counts the words that the candidates' compaction writes and compares the list with a sort.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "../paper_2411_01171_amd/csrc/k_select_search.h"

using namespace si;
typedef unsigned long long u64;

static int failures = 0, most = 0;

template <int KPL>
static void check(const std::vector<double>& score, int keep, const char* what) {
  const int n = (int)score.size();
  std::vector<u64> held(64 * KPL, 0);  // place i of lane l: block 64 i + l
  for (int j = 0; j < n; ++j) held[j] = order_key(score[j]);
  unsigned top = 0;
  for (u64 k : held) top = std::max(top, (unsigned)(k >> 32));
  auto tally = [&](auto pred) { return (int)std::count_if(held.begin(), held.end(), pred); };
  constexpr int WAYS = KPL <= 4 ? 4 : 2;
  UpperBounds b = upper_bounds<WAYS>(top, n, keep, KPL > 1 ? 64 : 0, [&](unsigned c) { return tally([&](u64 k) { return (unsigned)(k >> 32) >= c; }); });
  u64 least = (u64)b.lo << 32;
  bool exact = b.n_lo == keep;
  int need_equal = 0;
  if (!exact) {
    u64 end = (u64)b.hi << 32;
    if (b.n_lo - b.n_hi <= 64) {
      std::vector<u64> mine;
      for (u64 k : held)
        if (is_candidate(k, least, end)) mine.push_back(k);
      most = std::max(most, (int)mine.size());
      if ((int)mine.size() != b.n_lo - b.n_hi) {
        ++failures;
        std::printf("%s: KPL %d, %d blocks, keep %d: %zu places for %d candidates\n", what, KPL, n, keep, mine.size(), b.n_lo - b.n_hi);
      }
      mine.resize(64);
      const int above = b.n_hi;
      narrow<4>(least, end, b.n_lo, b.n_hi, keep, 0, [&](u64 c) { return above + (int)std::count_if(mine.begin(), mine.end(), [&](u64 k) { return k >= c; }); });
    } else {
      narrow<WAYS>(least, end, b.n_lo, b.n_hi, keep, 0, [&](u64 c) { return tally([&](u64 k) { return k >= c; }); });
    }
    exact = b.n_lo == keep;
    need_equal = keep - b.n_hi;
  }
  std::vector<int> order(n);
  for (int j = 0; j < n; ++j) order[j] = j;
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return held[x] > held[y]; });
  std::vector<bool> want(n, false);
  for (int i = 0; i < keep; ++i) want[order[i]] = true;
  int equal = 0;
  for (int j = 0; j < 64 * KPL; ++j) {
    const bool take = exact ? held[j] >= least : held[j] > least || (held[j] == least && equal++ < need_equal);
    if (take != (j < n && want[j])) {
      ++failures;
      std::printf("%s: KPL %d, %d blocks, keep %d: block %d\n", what, KPL, n, keep, j);
      return;
    }
  }
}

static void check(const std::vector<double>& score, int keep, int blocks, const char* what) {  // `blocks`: with those that hold no counted key
  if (blocks <= 64) check<1>(score, keep, what);
  else if (blocks <= 128) check<2>(score, keep, what);
  else if (blocks <= 256) check<4>(score, keep, what);
  else if (blocks <= 512) check<8>(score, keep, what);
  else check<16>(score, keep, what);
}

int main() {
  std::mt19937_64 rng(20);
  auto normal = [&] {  // sum of uniforms: the same on every library
    double s = -6;
    for (int i = 0; i < 12; ++i) s += (double)(rng() >> 11) * 0x1p-53;
    return s;
  };
  const int settings[][3] = {  // blocks, of which count, keep
      {70, 70, 35}, {72, 72, 36}, {80, 80, 60}, {100, 100, 90}, {128, 128, 64}, {129, 129, 65}, {144, 144, 72}, {300, 60, 30}, {300, 300, 200},
      {400, 400, 200}, {513, 513, 260}, {900, 100, 80}, {900, 900, 450}, {900, 900, 890}, {1024, 1024, 512}, {64, 64, 32}, {33, 33, 16}, {500, 2, 1}};
  for (auto& s : settings)
    for (int run = 0; run < 64; ++run) {
      std::vector<double> a(s[1]), wide(s[1]), ties(s[1]), low(s[1]);
      for (int j = 0; j < s[1]; ++j) {
        a[j] = normal();
        wide[j] = std::ldexp(normal(), (int)(rng() % 120) - 60);
        ties[j] = (double)(rng() % 3) - 1.0;
        low[j] = rng() % 2 ? -INFINITY : rng() % 8 ? normal() : NAN;
      }
      check(a, s[2], s[0], "normal");
      check(wide, s[2], s[0], "wide");
      check(ties, s[2], s[0], "ties");
      check(low, s[2], s[0], "not finite");
    }
  std::printf("%d failures, %d words at most\n", failures, most);
  return failures || most > 64;
}
