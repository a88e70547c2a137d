// Whether two heads of a call on queries and keys lie on one place.  Host arithmetic only, apart from the call so that a test can compile
// it by itself.  Internal: not part of the C ABI.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <numeric>

// counts[0] x counts[1] x counts[2] runs of `bytes` bytes, steps[i] bytes apart
struct LqRuns {
  uintptr_t at;
  int64_t steps[3], counts[3], bytes;
};

enum LqPlaces { LQ_APART = 0, LQ_SHARED = 1, LQ_ENTANGLED = 2 };      // entangled: not told within the steps below

// Whether c + the sum of step[i] x[i], lo[i] <= x[i] <= hi[i], falls into [low, high] for some whole x.  Steps in falling order of
// magnitude: what the later ones reach leaves an x few values where layouts are nested (about 0.1 us for an output inside a
// projection's rows).  Where it has many, what their steps have in common may settle it; the bound only meets layouts whose dimensions run
// through one another many times.
struct LqPlaceSearch {
  static constexpr int MAX_TERMS = 6, MAX_NODES = 1 << 16;
  struct Term {
    int64_t step, lo, hi;
  } term[MAX_TERMS];
  int64_t rest_lo[MAX_TERMS + 1], rest_hi[MAX_TERMS + 1], common[MAX_TERMS + 1], low, high;
  int n = 0, nodes = 0;

  void add(int64_t step, int64_t lo, int64_t hi) {
    if (step == 0 || (lo == 0 && hi == 0)) return;
    if (step < 0) { step = -step; std::swap(lo, hi); lo = -lo; hi = -hi; }
    term[n++] = {step, lo, hi};
  }
  static int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && a < 0); }
  LqPlaces run(int64_t c, int64_t from, int64_t to) {
    low = from; high = to;
    std::sort(term, term + n, [](const Term& a, const Term& b) { return a.step > b.step; });
    rest_lo[n] = rest_hi[n] = common[n] = 0;
    for (int i = n - 1; i >= 0; --i) {
      rest_lo[i] = rest_lo[i + 1] + term[i].step * term[i].lo;
      rest_hi[i] = rest_hi[i + 1] + term[i].step * term[i].hi;
      common[i] = std::gcd(common[i + 1], term[i].step);
    }
    return look(c, 0);
  }
  LqPlaces look(int64_t c, int i) {
    if (c + rest_hi[i] < low || c + rest_lo[i] > high) return LQ_APART;
    if (i == n) return LQ_SHARED;
    const Term& t = term[i];
    const int64_t first = std::max(t.lo, -floor_div(c + rest_hi[i + 1] - low, t.step));
    const int64_t last = std::min(t.hi, floor_div(high - c - rest_lo[i + 1], t.step));
    // c and a multiple of the common divisor
    if (last - first > 3 && floor_div(high - c, common[i]) < -floor_div(c - low, common[i])) return LQ_APART;
    for (int64_t x = first; x <= last; ++x) {
      if (++nodes > MAX_NODES) return LQ_ENTANGLED;
      const LqPlaces p = look(c + t.step * x, i + 1);
      if (p != LQ_APART) return p;
    }
    return LQ_APART;
  }
};

// From the first to behind the last byte, counted from `at`.  False: more than 2^60 bytes, which lie in no memory; below that no sum here
// leaves 64 bits.
static inline bool lq_runs_reach(const LqRuns& r, int64_t& lo, int64_t& hi) {
  double sum = (double)r.bytes;
  for (int i = 0; i < 3; ++i) sum += (double)(r.counts[i] - 1) * (double)(r.steps[i] < 0 ? -r.steps[i] : r.steps[i]);
  if (sum > 0x1p60) return false;
  lo = 0;
  hi = r.bytes;
  for (int i = 0; i < 3; ++i) (r.steps[i] < 0 ? lo : hi) += r.steps[i] * (r.counts[i] - 1);
  return true;
}
// two runs of one set
static inline LqPlaces lq_runs_collide(const LqRuns& r) {
  int64_t lo, hi;
  if (!lq_runs_reach(r, lo, hi)) return LQ_SHARED;
  // nested, each dimension's step as long as all that lies within it: apart (0.03 us; the search below takes 0.1)
  int order[3] = {0, 1, 2};
  const auto size = [&](int i) { return r.counts[i] < 2 ? 0 : r.steps[i] < 0 ? -r.steps[i] : r.steps[i]; };
  std::sort(order, order + 3, [&](int i, int j) { return size(i) < size(j); });
  int64_t reach = r.bytes;
  bool nested = true;
  for (int i : order) {
    nested = nested && (r.counts[i] < 2 || size(i) >= reach);
    reach += size(i) * (r.counts[i] - 1);
  }
  if (nested) return LQ_APART;
  for (int k = 0; k < 3; ++k) {                                // the first dimension that tells them apart
    if (r.counts[k] < 2) continue;
    if (r.steps[k] == 0) return LQ_SHARED;
    LqPlaceSearch s;
    s.add(r.steps[k], 1, r.counts[k] - 1);
    for (int i = k + 1; i < 3; ++i) s.add(r.steps[i], 1 - r.counts[i], r.counts[i] - 1);
    const LqPlaces p = s.run(0, 1 - r.bytes, r.bytes - 1);
    if (p != LQ_APART) return p;
  }
  return LQ_APART;
}
// a run of one set and a run of the other
static inline LqPlaces lq_runs_meet(const LqRuns& a, const LqRuns& b) {
  int64_t a_lo, a_hi, b_lo, b_hi;
  if (!lq_runs_reach(a, a_lo, a_hi) || !lq_runs_reach(b, b_lo, b_hi)) return LQ_SHARED;
  const int64_t apart = (int64_t)(b.at - a.at);
  if (apart + b_lo >= a_hi || apart + b_hi <= a_lo) return LQ_APART;
  LqPlaceSearch s;
  for (int i = 0; i < 3; ++i) {
    if (a.steps[i] == b.steps[i]) {                            // only the difference counts
      s.add(a.steps[i], 1 - a.counts[i], b.counts[i] - 1);
    } else {
      s.add(a.steps[i], 1 - a.counts[i], 0);
      s.add(b.steps[i], 0, b.counts[i] - 1);
    }
  }
  return s.run(apart, 1 - b.bytes, a.bytes - 1);
}
