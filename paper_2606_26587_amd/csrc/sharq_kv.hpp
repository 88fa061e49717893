// Indexing of the paged key/value cache and the work split of its attention.
// Plain C++ (constexpr functions run on both sides), so that a host test can
// replay a launch and check every index against its buffer.
#pragma once

#include <stdint.h>

namespace sharq {

// Buffers and sizes of a cache, as the kernels take them.  A cache row is one
// token of one key/value head; row (page * heads + head) * page_size + slot.
// Row numbers fit 32 bits (checked at the call), byte offsets need 64.
struct KvCacheArgs {
  uint8_t *k, *v;
  uint8_t *ks, *vs;   // E8M0 scales (MXFP4)
  int pages, heads, page_shift;
};

// The sequences of a call.
struct KvBatchArgs {
  const int32_t *offs, *lens, *table;
  int64_t ldt;
  int seqs, rows, max_len;
};

constexpr int kv_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Cache row of token t through a row of a page table, -1 when the page lies
// outside the pool.  t must be inside the table.
constexpr int kv_row(int page, int t, int pages, int heads, int head, int page_shift) {
  return page < 0 || page >= pages ? -1
                                   : (int)(((((int64_t)page * heads + head) << page_shift)) +
                                           (t & ((1 << page_shift) - 1)));
}

// The tiles of T tokens, cut from token t0 on, that rows at the positions
// p_lo..p_hi see of the tokens [t0, t1).  A row at p sees the tokens t <= p
// with p - t < window or t < sinks.  Tiles of the sinks come first, then those
// of the window: tile i of n starts at token t0 + T * (i < ns ? i : i - ns + jf).
struct KvSpan {
  int ns, jf, n;
  int low, hi;   // some row sees t  <=>  t < hi and (t >= low or t < sinks)
};

constexpr KvSpan kv_span(int t0, int t1, int p_lo, int p_hi, int window, int sinks, int T) {
  KvSpan s{0, 0, 0, 0, 0};
  s.hi = p_hi < t1 - 1 ? p_hi + 1 : t1;
  s.low = p_lo >= window ? p_lo - window + 1 : 0;
  if (s.hi <= t0) return s;
  const int se = sinks < s.hi ? sinks : s.hi;
  if (se > t0) s.ns = (se - t0 + T - 1) / T;
  const int first = s.low > t0 ? (s.low - t0) / T : 0;
  s.jf = first > s.ns ? first : s.ns;
  const int end = (s.hi - t0 + T - 1) / T;
  s.n = s.ns + (end > s.jf ? end - s.jf : 0);
  return s;
}

constexpr int kv_tile_start(const KvSpan& s, int t0, int i, int T) {
  return t0 + T * (i < s.ns ? i : i - s.ns + s.jf);
}

}  // namespace sharq
