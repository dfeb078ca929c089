// Debug build: the buffers that callers hand to a call (host arithmetic).
//
// A call only enqueues and may be captured, so that its buffers stay in the table of ranges (debug_check.cuh) when it
// returns.  But a range is to be no larger than the buffer that is there now: the buffers of a call take the place of kept
// ones that they overlap (memory that was freed and handed out again, or a part of an older buffer), and a handle's
// go when it is destroyed.  Where there are more than kRoom, the one that was not used for the longest time makes room.
#pragma once
#include <stdint.h>

namespace hadfl {

class DebugKept {
 public:
  static constexpr int kRoom = 16;
  struct Range {
    uint64_t lo, hi;
    bool operator==(const Range &o) const { return lo == o.lo && hi == o.hi; }
    bool meets(const Range &o) const { return lo < o.hi && o.lo < hi; }
  };

  // The n buffers of one call of `owner` (which may overlap each other).  Returns whether the table has changed.
  bool keep(const void *owner, const Range *call, int n) {
    bool changed = false;
    ++now_;
    for (Kept &k : kept_) {
      bool meets = false, is_of_call = false;
      for (int i = 0; i < n; ++i) {
        meets |= k.used && k.range.meets(call[i]);
        is_of_call |= k.range == call[i];
      }
      if (!meets || is_of_call) continue;
      k = Kept();
      changed = true;
    }
    for (int i = 0; i < n; ++i) {
      if (call[i].lo >= call[i].hi) continue;
      Kept *at = kept_;
      for (Kept &k : kept_) {
        if (k.used && k.owner == owner && k.range == call[i]) {
          at = &k;
          break;
        }
        if (k.used < at->used) at = &k;
      }
      if (!(at->used && at->owner == owner && at->range == call[i])) {
        *at = Kept{call[i], owner, 0};
        changed = true;
      }
      at->used = now_;
    }
    return changed;
  }
  void forget(const void *owner) {
    for (Kept &k : kept_)
      if (k.owner == owner) k = Kept();
  }
  // Calls f(range) for each.
  template <typename F>
  void each(F &&f) const {
    for (const Kept &k : kept_)
      if (k.used) f(k.range);
  }

 private:
  struct Kept {
    Range range = {0, 0};
    const void *owner = nullptr;
    uint64_t used = 0;  // number of the call, 0: free
  };
  Kept kept_[kRoom];
  uint64_t now_ = 0;
};

}  // namespace hadfl
