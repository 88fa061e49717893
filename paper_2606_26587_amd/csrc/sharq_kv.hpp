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

// ---------------------------------------------------------------------------
// Launches of the append and the read-back
// ---------------------------------------------------------------------------

constexpr int kAppendThreads = 128, kReadThreads = 128;

// Workgroups of a row: a thread takes 16 values in the append, 8 in the read-back.
constexpr int kv_append_parts(int q_heads, int heads, int D) {
  return ((q_heads + 2 * heads) * (D / 16) + kAppendThreads - 1) / kAppendThreads;
}
constexpr int kv_read_parts(int heads, int D) { return (2 * heads * (D / 8) + kReadThreads - 1) / kReadThreads; }

// A launch has fewer than 2^32 threads.
constexpr bool kv_launches(int64_t blocks, int threads) { return blocks <= 0xFFFFFFFFll / threads; }

// ---------------------------------------------------------------------------
// Work split of the attention
// ---------------------------------------------------------------------------

constexpr int kAttnTile = 64;    // tokens of a key/value tile where rows are many
constexpr int kAttnRows = 128;   // rows (token x query head of a key/value head) of a tile there

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// `chunks` workgroups share the tokens of each of `tiles` row tiles, `chunk_tiles`
// key/value tiles each.
struct AttnSplit {
  int tiles, chunks, chunk_tiles;
};

struct AttnPlan {
  int few;          // 16-row tiles of the few-row kernel (1, 2, 4); 0: the kernel for many rows
  bool shared;      // the prefix is read for all sequences together
  AttnSplit own, prefix;
  int slots;        // partial results of a row; 0: none, results are final
  bool mixed;       // sequences of few rows and of many, each by its kernel
};

// Splits kv_tiles of each of `units` workgroups so that about `want` workgroups
// run, each over a multiple of `least` tiles.  kv_tiles follows from the host's
// bounds: sequences far shorter than max_len fall into the first parts, and the
// workgroups of the others end at once.  4 single tokens over 4000, 32 and 8 heads
// of 128 in bf16: 17.4 us with max_len 4000, 23.4 with 16384, 38.6 with 131072; a
// prompt of 512 15.5 us, 27.7 (and 34 MB of workspace) with max_len 8192.
constexpr AttnSplit attn_split(int64_t tiles, int64_t units, int64_t kv_tiles, int64_t want, int least) {
  int64_t chunks = units > 0 ? want / units : 1;
  if (chunks > ceil_div(kv_tiles, least)) chunks = ceil_div(kv_tiles, least);
  if (chunks < 1) chunks = 1;
  int64_t each = ceil_div(ceil_div(kv_tiles, chunks), least) * least;
  if (each < least) each = least;
  chunks = kv_tiles > 0 ? ceil_div(kv_tiles, each) : 1;
  return {(int)tiles, (int)chunks, (int)each};
}

constexpr AttnPlan attn_plan(int64_t seqs, int64_t rows, int64_t max_rows, int64_t max_len, int heads, int group, int D,
                             bool mx, int64_t window, int64_t sinks, int64_t prefix_len) {
  AttnPlan p{};
  if (max_rows > rows) max_rows = rows;
  // a window leaves little of a prefix, and rows that see different parts of it
  p.shared = prefix_len > 0 && window >= max_len;
  const int64_t r = max_rows * group, own = max_len - (p.shared ? prefix_len : 0);
  // The kernel for few rows up to 16, and up to 32 or 64 where it is the faster one.  In it and in the kernel for many:
  // bf16, heads of 128, 16 x 8 tokens of 4 query heads over 8000 87 and 81 us, 64 x 5 over 600 29 and 25, 1 x 8 over
  // 4000 13.6 and 14.4; heads of 64, 2 x 8 over 16000 19 and 23, 16 x 12 over 8000 62 and 58; MXFP4, heads of 64,
  // 16 x 12 39 and 53.  (64 rows' states over heads of 128 fill the registers.)
  p.few = r <= 16 ? 1 : r <= 32 && (D == 64 || mx) ? 2 : r <= 64 && D == 64 && mx ? 4 : 0;
  // tokens that a tile of rows sees at most: its window and its own positions, and the sinks
  const int64_t span = p.few ? max_rows : kAttnRows / group + 2;
  const int64_t w = window < max_len ? window + span : own, part = w < own ? w : own;
  const int64_t s = window < max_len ? (sinks < own - part ? sinks : own - part) : 0;
  if (p.few) {
    const int tok = mx ? 64 : 32;
    const int64_t kv = part > 0 ? ceil_div(part, tok) + (part < own ? 1 : 0) + ceil_div(s, tok) : 0;
    // One round of workgroups where a wavefront has few turns of its tiles.  Where it has many, and the kernel's states
    // leave room for three workgroups a CU, four rounds: then what sequences of different lengths leave idle counts for
    // more than starting up and joining.  One round against four, 8 heads: single tokens in bf16, 8 x 8191 44.8 and
    // 47.2 us, 64 x 1000 40.3 and 45.1, 64 x 4000 135 and 124, 24 x 32768 502 and 420; 5 tokens a sequence, 20 rows
    // of heads of 64, over 16 x 16000 98.8 and 82.6.  Beside a shared prefix's workgroups: one round.
    const bool lean = p.few == 1 || (p.few == 2 && D == 64);
    const int64_t units = seqs * heads, turns = units * ceil_div(kv, 4);
    // Where one round leaves a third of the chip idle, two: 33 x 1500 single tokens in bf16 47.2 and 36.9 us, 40 x 1500
    // 45.6 and 39.9; 33 x 8 tokens over 5000 in MXFP4 68.1 and 55.1.  (With 480 of 512 places taken the same loses 10%.)
    const bool idle = units > 256 && units <= 341 && turns >= (lean ? 3000 : 4000);
    const int want = p.shared ? 512 : lean && turns >= 6144 ? 2048 : idle ? 1024 : mx && p.few == 1 ? 768 : 512;
    p.own = attn_split(1, units, kv, want, 4);
  } else {
    // no sequence has more than max_rows rows, and all together have no more than rows
    const int64_t most = seqs * ceil_div(r, kAttnRows), packed = rows * group / kAttnRows + seqs;
    const int64_t tiles = most < packed ? most : packed;
    const int64_t kv = part > 0 ? ceil_div(part, kAttnTile) + (part < own ? 1 : 0) + ceil_div(s, kAttnTile) : 0;
    // About as many workgroups as the chip holds (2 a CU; heads of 64: 3): 500 rows over 12000 tokens, 4 heads of 64:
    // 70.8 us with 512, 66.2 with 1024; of 128: 101 and 112, where the partial results weigh more.  Sequences of
    // different lengths fill half of their last tiles: 32 x up to 17 tokens over 8000, 4 x 8 heads of 128, 130 us with
    // whole last tiles counted, 106 with halves; 6 x 100 over 6000, 8 x 4 heads, 73 and 63.
    int64_t likely = rows * group / kAttnRows + seqs / 2 + 1;
    likely = likely < seqs ? seqs : likely;
    const int64_t units = (likely < tiles ? likely : tiles) * heads;
    p.own = attn_split(tiles, units, kv, D == 64 ? 1024 : 512, 4);
    // Not where the partial results take longer than what the split saves of the longest walk: ns of a tile, alone on its
    // CU or not, and of a row and head's partial result, written and read.  A prompt of 1024, 32 query heads of 128:
    // 36.0 us split in two, 27.5 whole; 4 x 300, 16 query heads, 19.0 in five parts, 11.9 whole.
    const int64_t alone = D == 64 ? 1250 : 1400, among = D == 64 ? 1900 : 2100;
    const int64_t whole = kv * (units > 256 ? among : alone);
    const int64_t split = p.own.chunk_tiles * (units * p.own.chunks > 256 ? among : alone) + 4000 +
                          rows * heads * group * p.own.chunks * (D + 2) * 2 * 4 / 4500;
    if (whole <= split) p.own = attn_split(tiles, units, kv, 1, 4);
    // The mean below two thirds of the longest: some sequences may have a token each, on which the kernel for many rows
    // spends a whole tile's dequantization.  How many do, the host does not know, and need not: the kernel for many rows
    // alone and both in one launch, in MXFP4, 32 and 8 heads of 128: a prompt of 2000 and 63 single tokens over 4000 152
    // and 99 us, 6 prompts of 1000 and 4 single tokens over 8000 (mean 0.6) 171 and 119, 16 of 1000 and 16 over 4000 216
    // and 209, but 2 of 2000 and 6 over 4000 95 and 104; prompts alone, whose lengths differ, 20 of 125 to 2000 302 and
    // 300, 1000, 400 and 300 29.2 and 28.9, heads of 64 185 and 186.  (bf16: 240 and 226, but a chunk of 512 and 31
    // single tokens over 8000 238 and 251.)
    p.mixed = mx && !p.shared && p.own.chunks == 1 && 3 * rows < 2 * seqs * max_rows;
  }
  p.slots = p.own.chunks > 1 ? p.own.chunks : 0;
  if (p.shared) {
    const int64_t tiles = ceil_div(rows * group, kAttnRows);
    // 64 tokens behind 8192, 400 of their own each: 49.6 us with 256 workgroups, 49.8 with 384, 56.2 with 512; 44.5 with
    // 192, but 16 behind 32768 then 45.2 against 41.4 (384: 42.4), and 40 x 4 behind 4096 in MXFP4 33.3 against 29.8
    const int64_t kv = ceil_div(prefix_len, kAttnTile), units = tiles * heads;
    p.prefix = attn_split(tiles, units, kv, 256, 2);
    // Where that leaves long walks (then the partial results weigh less), twice as many: 32 x up to 32 tokens behind 4096,
    // 32 and 8 heads of 128, 94.7 and 82.8 us, behind 16384 339 and 258; 4 single tokens behind 61440 in MXFP4 48.4 and
    // 35.2; 256 behind 16384 118 and 122, in MXFP4 106 and 103.  (8 x 100 behind 2048, 32 tiles: 39.5 and 45.2.)
    if (kv >= 48 && p.prefix.chunk_tiles >= 28) p.prefix = attn_split(tiles, units, kv, 512, 2);
    p.slots = p.own.chunks + p.prefix.chunks;
  }
  return p;
}

// Bytes of the softmax states of `items` rows and heads in `slots` slots (the
// partial outputs lie behind them, 16-byte aligned).
constexpr int64_t attn_ml_bytes(int64_t items, int slots) { return ceil_div(items * slots * 8, 16) * 16; }
constexpr int64_t attn_workspace(int64_t items, int slots, int D) {
  return slots ? attn_ml_bytes(items, slots) + items * slots * D * 4 : 0;
}

}  // namespace sharq
