// The token window of an attention call, as the host and the kernels take it.
#pragma once

#include <cstdint>

namespace ws {

// Token window of an attention call.  The visible tokens under the call's mask,
// in order, are the timeline; row i of the call sits at index t = t0 + i and sees
// the keys j with (j > t - window or j < sinks) and j < t + ahead (1: causal).  The
// page list then carries each page's first index: entry y = valid | start << 7.
struct TokenWindow {
  int32_t on;       // 0: every key of the page list is visible to every row
  int32_t ahead;    // 1 or kNoWindow
  int32_t t0;
  int32_t window;   // 1 .. kNoWindow
  int32_t sinks;
  int32_t n_keys;   // tokens of the timeline
};
constexpr int32_t kMaxTimeline = 1 << 24;  // tokens that page entries can index
constexpr int32_t kNoWindow = 1 << 30;     // (a timeline and 2^20 rows past it stay below 2^31 with it)

// The pages of a query class, or of a query tile, within a window call's list: its
// first head_pages entries and, `skip` entries further, the others of `count`.
struct ClassPages {
  int32_t head_pages, skip, count;
};

}  // namespace ws
