// Whether two tensors of heads share memory.  Plain C++, so that it is tested
// without a GPU.
#pragma once

#include <cstdint>

namespace mpt {

// [tokens][heads] runs of contiguous bytes; steps in bytes, positive where there
// is more than one of the axis.
struct HeadRuns {
  uintptr_t at;
  int64_t run;
  int64_t n[2], step[2];  // tokens and heads
};

namespace overlap_detail {

using wide = __int128;  // 2^31 tokens times a stride of 2^40 bytes

struct Term {  // i step, lo <= i <= hi
  wide step, lo, hi;
};

inline wide floor_div(wide a, wide b) { return a / b - (a % b < 0); }  // b > 0

// Whether low < x + a sum of the terms from k on < high, for some choice of
// them; false also where that takes more than `left` steps to find out.
inline bool reaches(wide x, const Term* t, int k, int n, wide low, wide high, int& left) {
  if (k == n) return low < x && x < high;
  wide lo = 0, hi = 0;  // of the later terms' sum
  for (int j = k + 1; j < n; ++j) lo += t[j].lo * t[j].step, hi += t[j].hi * t[j].step;
  wide first = floor_div(low - x - hi, t[k].step) + 1, last = -floor_div(-(high - x - lo), t[k].step) - 1;
  if (first < t[k].lo) first = t[k].lo;
  if (last > t[k].hi) last = t[k].hi;
  for (wide i = first; i <= last; ++i) {
    if (--left < 0) return false;
    if (reaches(x + i * t[k].step, t, k + 1, n, low, high, left)) return true;
  }
  return false;
}

}  // namespace overlap_detail

// A shared byte is a pair of runs that begin less than a run apart: a difference
// of addresses and of multiples of steps, looked for from the largest step down,
// so that tensors of ordinary layouts take a handful of tries.  Exact, but that
// layouts of many tokens with odd steps (1,024 tries) are taken to be apart.
inline bool heads_overlap(const HeadRuns& a, const HeadRuns& b) {
  using namespace overlap_detail;
  const HeadRuns* const both[2] = {&a, &b};
  Term t[4];
  wide run[2];
  int n = 0;
  for (int s = 0; s < 2; ++s) {
    run[s] = both[s]->run;
    bool taken[2] = {both[s]->n[0] == 1, both[s]->n[1] == 1};
    for (int r = 0; r < 2; ++r)  // axes whose entries follow one another are one longer run
      for (int i = 0; i < 2; ++i)
        if (!taken[i] && both[s]->step[i] == run[s]) run[s] *= both[s]->n[i], taken[i] = true;
    for (int i = 0; i < 2; ++i) {
      if (taken[i]) continue;
      const wide most = both[s]->n[i] - 1;
      int j = 0;
      while (j < n && t[j].step != both[s]->step[i]) ++j;
      if (j == n) t[n++] = {both[s]->step[i], 0, 0};
      if (s == 0) t[j].lo -= most;
      else t[j].hi += most;
    }
  }
  for (int i = 1; i < n; ++i)  // larger steps first
    for (int j = i; j > 0 && t[j].step > t[j - 1].step; --j) {
      const Term x = t[j];
      t[j] = t[j - 1], t[j - 1] = x;
    }
  int left = 1024;
  return reaches((wide)b.at - (wide)a.at, t, 0, n, -run[1], run[0], left);
}

}  // namespace mpt
