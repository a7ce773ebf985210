// Equal shares of the steps of items laid end to end, one to a CTA (the gradient of
// attention, mha_backward.cu).  Whole numbers alone, the same on the host.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define ACID_HD __host__ __device__ __forceinline__
#else
#define ACID_HD inline
#endif

namespace acid {

// The items are the slots of one head after another; those from `full` on are shared
// out.  upto(slot): steps of a head's slots up to and with this one.  An item's steps fit
// 32 bits, a head's do not (2^20 rows, 32 query heads on one key head: 2^31).
template <class Upto>
struct StepShares {
  Upto upto;
  int slots, full, shares;
  int64_t total, base, work;  // steps of a head, those before the shared ones, the shared ones
  ACID_HD StepShares() : upto(), slots(0), full(0), shares(1), total(0), base(0), work(0) {}
  ACID_HD StepShares(const Upto& u, int heads, int slots_, int full_, int ctas, int least)
      : upto(u), slots(slots_), full(full_), total(u(slots_ - 1)) {
    base = full / slots * total + before(full % slots);
    work = heads * total - base;
    const int64_t most = work / least;
    shares = most < 1 ? 1 : most < ctas ? (int)most : ctas;
  }
  // Steps of a head's slots before this one.
  ACID_HD int64_t before(int slot) const { return slot > 0 ? upto(slot - 1) : 0; }
  // First step of share c, and the one past the last of share c - 1.
  ACID_HD int64_t bound(int64_t c) const { return base + work * c / shares; }
  // The item that the first step of share c lies in, and that item's first step.
  ACID_HD void begin(int c, int& item, int64_t& first) const {
    if (c == 0) {  // (with those before it that have no steps)
      item = full;
      first = base;
      return;
    }
    const int64_t from = bound(c);
    const int head = (int)(from / total);
    const int64_t rest = from - head * total;
    int lo = 0, hi = slots - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (upto(mid) > rest) hi = mid;
      else lo = mid + 1;
    }
    item = head * slots + lo;
    first = head * total + before(lo);
  }
};

}  // namespace acid
