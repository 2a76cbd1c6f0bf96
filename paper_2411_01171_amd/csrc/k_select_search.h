// The search for the `keep`-th largest of a list of scores, over their order as unsigned integers.  Plain arithmetic around
// the caller's counts, so that host code can run it as well.
#pragma once
#include <cmath>

namespace si {

// Order of float64 as unsigned integers: NaN as -infinity, -0 as +0.  The least key is -infinity's, 0x000fffff ffffffff; 0 stands
// for a place without a score.
__host__ __device__ __forceinline__ unsigned long long order_key(double x) {
  if (!(x == x)) x = -INFINITY;
  const unsigned long long b = __builtin_bit_cast(unsigned long long, x + 0.0);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

// Narrows [lo, hi) to the largest T with count(T) = (number of values >= T) >= need, where count(lo) = n_lo >= need > n_hi =
// count(hi).  Ends with hi = lo + 1, or as soon as count(lo) is `need`, or when no more than `few` values lie in [lo, hi).
// WAYS parts per step: 4 where a count is nearly all latency (a few ballots), 2 where it is work.
template <int WAYS, class U, class Count>
__host__ __device__ __forceinline__ void narrow(U& lo, U& hi, int& n_lo, int& n_hi, int need, int few, Count count) {
  while (hi - lo > 1 && n_lo != need && n_lo - n_hi > few) {
    const U part = hi - lo > WAYS ? (hi - lo) / WAYS : 1;
    int n[WAYS];
#pragma unroll
    for (int i = 1; i < WAYS; ++i) n[i] = count(lo + part * i);  // past the end: too few
    const U base = lo;
#pragma unroll
    for (int i = 1; i < WAYS; ++i)  // counts fall with i
      if (n[i] >= need) { lo = base + part * i; n_lo = n[i]; }
#pragma unroll
    for (int i = WAYS - 1; i > 0; --i)
      if (n[i] < need) { hi = base + part * i; n_hi = n[i]; }
  }
}

// [lo, hi): upper words (of 32 bits) between which the `keep`-th largest key's lies; n_lo, n_hi: keys from there on.
struct UpperBounds {
  unsigned lo, hi;
  int n_lo, n_hi;
};

// `n` keys (n > keep), the largest upper word `top`; upper(c) counts the keys whose upper word is at least c.  From eight binades
// below the largest on first: most lists have their threshold there.  lo is at least 1, below every score's upper word and above
// that of a place without one.
template <int WAYS, class Count>
__host__ __device__ __forceinline__ UpperBounds upper_bounds(unsigned top, int n, int keep, int few, Count upper) {
  constexpr unsigned kBinades = 8u << 20;
  UpperBounds b{1u, top + 1, n, 0};  // top is at most the infinity's
  const unsigned first = top > kBinades ? top - kBinades : top / 2 + 1;
  const int c = upper(first);
  if (c >= keep) { b.lo = first; b.n_lo = c; }
  else { b.hi = first; b.n_hi = c; }
  narrow<WAYS>(b.lo, b.hi, b.n_lo, b.n_hi, keep, few, upper);
  return b;
}

// Whether a place's key is among those left: with `least` of 2^32 and more, as upper_bounds leaves it, no place without a score
// is, so that there are n_lo - n_hi of them.
__host__ __device__ __forceinline__ bool is_candidate(unsigned long long key, unsigned long long least, unsigned long long end) {
  return key >= least && key < end;
}

}  // namespace si
