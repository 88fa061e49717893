// Causal attention over the paged key/value cache, with a sliding window and
// first tokens that stay visible (sinks).
//
// For a row at position p, o = sum_t w_t v_t over the tokens t <= p with
// p - t < window or t < sinks, w = softmax(scale q.k).  One pass over the
// tokens with the running maximum m and sum l of the softmax:
//   m' = max(m, s_t), l' = l e^(m - m') + sum e^(s_t - m'), o' likewise.
//
// The rows of a key/value head's query heads are worked on together: row r of a
// tile is token r / G, query head r % G of the G heads that share the cached
// head, so a token's keys and values are read once for all of them.
//
// Both products are computed transposed, S^T = K Q^T and O^T = V^T P^T, with
// 32x32x16 bf16 MFMAs.  A lane then holds one row of S (a column of S^T) and the
// same row of O: maxima, sums and the rescaling by e^(m - m') need no broadcast,
// and the accumulator registers of S^T, rounded to bf16, are the operand of the
// second product as they stand, when the eight k slots of a lane half h are
// taken as the tokens {4h..4h+3, 8+4h..8+4h+3} of each 16.  The matching V^T
// operand comes from row-major V in LDS through the transposing LDS read.
//
// P is rounded to bf16 for the second product (V is bf16, and so is the output);
// m, l, o and the sum of P stay in fp32.
//
// A workgroup holds 128 rows, 32 a wavefront (o 64, q 32, S^T 32 registers of 256:
// two wavefronts a SIMD, of two workgroups that run apart, so one's exponentials
// can run beside the other's products), and walks tiles of 64 tokens in two LDS
// stages: while one is worked on, the next is on its way, bf16 straight from
// global memory to LDS; E4M3, and of MXFP4 the next two, through registers, from
// where it becomes bf16 once for all rows.  Rows of consecutive tokens share the tiles:
// with 4 query heads a key/value head a tile is 32 tokens, so little of a causal
// or windowed tile is masked, and masks are formed only in tiles that need one.
//
// Measured (8192 tokens, 32 query and 8 key/value heads of 128, causal): 532 to 546
// us across boxes, 1.02 PFLOP/s, 0.84 of what a library bf16 product of 8192^3 reaches on the same
// card.  The matrix cores are busy half of the cycles and so is the VALU; what
// bounds it is power: on zeros the same launch takes 424 us.  Tiles of 32 tokens
// with three wavefronts a SIMD (586 us), the first half's exponentials beside the
// second half's products (544, and with the maximum left out 546 against 540),
// halves of masked tiles skipped (571) and raised priority around the products
// (550) were measured and not kept.  Heads of 64: 830 TFLOP/s, the exponentials
// weigh twice as much.  An MXFP4 cache costs 2.5% here (538 and 552), one in E4M3 6.5%
// (494 and 527): twice the registers and loads of MXFP4 on the way, the same conversions.

#pragma once

#include <type_traits>

#include "sharq_attn.hpp"

namespace sharq {

constexpr int kSchedMfma = 0x8, kSchedLdsRead = 0x100;   // kinds of instructions to the scheduler
constexpr int kT = kAttnTile;        // tokens of a key/value tile
constexpr int kRowsA = kAttnRows;    // rows of a workgroup: 32 a wavefront

// Sequence (and its rows) and tile of work unit `unit` of tiles of kRowsA rows, over the sequences of more than
// few_rows rows; false: none.
__device__ __forceinline__ bool find_tile(const KvBatchArgs& b, int group, int few_rows, int unit, int& seq, SeqRows& sr,
                                          int& tile) {
  const int lane = (int)(threadIdx.x & 63);
  int base = 0;
  for (int s0 = 0; s0 < b.seqs; s0 += 64) {
    const int s = s0 + lane;
    SeqRows r{0, 0, 0};
    if (s < b.seqs) r = seq_rows(b, s);
    const int n = r.n * group > few_rows ? (r.n * group + kRowsA - 1) / kRowsA : 0;
    int sum = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    const unsigned long long past = __ballot(base + sum > unit);
    if (past) {
      const int l = __builtin_ctzll(past);
      seq = s0 + l;
      sr.first = __builtin_amdgcn_readlane(r.first, l), sr.n = __builtin_amdgcn_readlane(r.n, l);
      sr.len = __builtin_amdgcn_readlane(r.len, l);
      tile = unit - base - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(n, l));
      return true;
    }
    base += __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// The rows of one tile: the sequences' own parts (ALL false: a tile's rows are
// of one sequence) or the shared prefix (ALL: rows of all sequences).
template <int D>
struct RowsLds {
  uint4 kv[2][2][kT * D / 8];   // two stages of keys and values
};

template <int D, int F, bool ALL>
__device__ __forceinline__ void attn_rows(const AttnArgs& a, int block, int tiles, int chunk_tiles, int first_slot,
                                          RowsLds<D>& shared) {
  constexpr bool MX = F == kKvMx, F8 = F == kKvF8, CODES = MX || F8;
  constexpr int kC = D / 8, kDT = D / 32;   // 16-byte chunks of a row, 32-wide tiles of D
  auto& lds = shared.kv;
  int* const lds_p = reinterpret_cast<int*>(&lds[0][0][0]);
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  // heads fastest: workgroups are dealt to the XCDs in turn, so each L2 sees few heads' keys and values.
  // Late tiles of a sequence, which see most tokens, first.
  const int head = block % a.c.heads;
  const int uc = block / a.c.heads, chunk = uc / tiles, unit = tiles - 1 - uc % tiles;
  const int rr = wave * 32 + (lane & 31);
  const unsigned group = (unsigned)a.group;   // rows times heads of a call fit 27 bits
  int seq = 0, rows, row_g, qh, p;                  // of this lane: row of the call, query head, position
  int p_lo, p_hi, w_lo, w_hi, t0, t1;               // positions of the workgroup's and the wavefront's rows; tokens
  if (ALL) {
    const int all = kv_clamp(a.b.offs[a.b.seqs], 0, a.b.rows), total = all * a.group, r0 = unit * kRowsA;
    if (r0 >= total) return;
    rows = total - r0 < kRowsA ? total - r0 : kRowsA;
    const unsigned r = (unsigned)(r0 + (rr < rows ? rr : rows - 1));
    row_g = (int)(r / group), qh = head * a.group + (int)(r % group);
    // Rows past the prefix see all of it, wherever they are.
    p = p_lo = p_hi = w_lo = w_hi = a.prefix_len;
    t0 = 0, t1 = a.prefix_len;
  } else {
    int tile;
    SeqRows sr;
    if (!find_tile(a.b, a.group, a.few_rows, unit, seq, sr, tile)) return;
    const int r0 = tile * kRowsA, total = sr.n * a.group;
    const int base = sr.len - sr.n;   // position of the sequence's first row
    rows = total - r0 < kRowsA ? total - r0 : kRowsA;
    const unsigned r = (unsigned)(r0 + (rr < rows ? rr : rows - 1));
    const int token = (int)(r / group);
    row_g = sr.first + token, qh = head * a.group + (int)(r % group), p = base + token;
    const unsigned wr = wave * 32 < rows ? wave * 32 : rows - 1, we = wave * 32 + 31 < rows ? wave * 32 + 31 : rows - 1;
    p_lo = base + (int)((unsigned)r0 / group), p_hi = base + (int)((unsigned)(r0 + rows - 1) / group);
    w_lo = base + (int)((r0 + wr) / group), w_hi = base + (int)((r0 + we) / group);
    t0 = a.t0, t1 = sr.len;
  }

  v8bf qf[D / 16];
  {
    const uint16_t* qp = a.q + (int64_t)row_g * a.ldq + (int64_t)qh * D + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) qf[i] = *reinterpret_cast<const v8bf*>(qp + 16 * i);
  }
  if (ALL) {   // unless a sequence has rows inside the prefix: then every lane looks for its row's sequence
    bool inside = false;
    for (int s = lane; s - lane < a.b.seqs; s += 64) {
      SeqRows sr{0, 0, 0};
      if (s < a.b.seqs) sr = seq_rows(a.b, s);
      inside |= __any(sr.n > 0 && sr.len - sr.n < a.prefix_len);
    }
    if (inside) {
      const int last = (int)((unsigned)(unit * kRowsA + rows - 1) / group);
      int s = find_seq(a.b, (int)((unsigned)(unit * kRowsA) / group));   // of the first row
      for (int at = s; at < a.b.seqs; at += 64) {   // past those that end at or before this lane's, 64 at a time
        const int end = at + lane < a.b.seqs ? a.b.offs[at + lane + 1] : 0x7FFFFFFF;
        for (int i = 0; i < 64; ++i) s += __builtin_amdgcn_readlane(end, i) <= row_g;
        if (__builtin_amdgcn_readlane(end, 63) > last) break;
      }
      const SeqRows sr = seq_rows(a.b, s < a.b.seqs ? s : a.b.seqs - 1);
      p = sr.len - sr.n + (row_g - sr.first);
      int lo = p, hi = p;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_xor(lo, d), w = __shfl_xor(hi, d);
        lo = u < lo ? u : lo, hi = w > hi ? w : hi;
      }
      w_lo = __builtin_amdgcn_readfirstlane(lo), w_hi = __builtin_amdgcn_readfirstlane(hi);
      if (lane == 0) lds_p[wave] = lo, lds_p[4 + wave] = hi;
      __syncthreads();
      p_lo = __builtin_amdgcn_readfirstlane(lds_p[0]), p_hi = __builtin_amdgcn_readfirstlane(lds_p[4]);
#pragma unroll
      for (int i = 1; i < 4; ++i) {
        const int u = __builtin_amdgcn_readfirstlane(lds_p[i]), w = __builtin_amdgcn_readfirstlane(lds_p[4 + i]);
        p_lo = u < p_lo ? u : p_lo, p_hi = w > p_hi ? w : p_hi;
      }
      __syncthreads();
    }
  }
  v16f o[kDT] = {};
  float m = kNoMax, l = 0.0f;

  if (wave * 32 >= rows) w_hi = -1;   // no rows: loads its share of the tiles, no more
  const KvSpan span = kv_span(t0, t1, p_lo, p_hi, a.window, a.sinks, kT);
  const int first = chunk * chunk_tiles, end = span.n < first + chunk_tiles ? span.n : first + chunk_tiles;
  // lane i: page of token i of a tile (of another that is seen where it is not: the load has no condition), and its
  // cache row, -1 where no row sees it (its page may hold anything)
  auto page_of = [&](int ti) {
    const int t = kv_tile_start(span, t0, ti, kT) + lane;
    return token_page(a, seq, t < span.hi ? t : span.hi - 1);
  };
  auto row_of = [&](int page, int ti) {
    const int t = kv_tile_start(span, t0, ti, kT) + lane;
    const bool seen = ti < end && t < span.hi && (t >= span.low || t < a.sinks);
    return seen ? kv_row(page, t, a.c.pages, a.c.heads, head, a.c.page_shift) : -1;
  };
  // A wavefront stages 16 tokens of a tile, which lie in one page: tiles start at multiples of 16.
  constexpr int kI = kC / 4, kRowsLoad = 64 / kC;   // bf16: 16-byte loads of a lane, keys or values; rows of a load
  uint32_t off[kI];   // this lane's place in the 16 tokens; the exchange of chunks is made here
#pragma unroll
  for (int i = 0; i < kI; ++i) {
    const int row = i * kRowsLoad + lane / kC;
    off[i] = (uint32_t)(row * D * 2 + 16 * (kv_chunk<D>(row, lane % kC) - row * kC));
  }
  // MXFP4: two tiles' codes and scales on their way, 32 values a lane: 16 tokens at one place of their rows, so that
  // they go to LDS over all banks.  A step of few rows is shorter than the way from HBM: with one tile on its way
  // 16 x 9 tokens, 4 query heads a key/value head, over 8000 took 80 us, with two 69; a prompt of 5759, heads of 64,
  // 210 and 191.
  // E4M3: 16 values a load, and the 16 tokens have one scale; one tile on its way, as two take the registers that the
  // products need (two prompts of 6000, 28 and 4 heads of 128: 512 us with two, 502 with one).
  constexpr int kW = F8 ? D / 64 : 1;
  struct Codes {
    uint4 k[kW], v[kW];
    uint32_t ks, vs;
  } ahead[CODES ? 2 : 1];
  const int mx_row = mx_token<D>(lane), mx_block = (lane >> 4) % (D / 32);
  const int mx_byte = mx_row * (D / 32) + mx_block;   // of the 16 tokens' scales; loaded as the dword that holds it
  auto load = [&](int at, int to) {
    const unsigned mine = (unsigned)(__ballot(at >= 0) >> (16 * wave)) & 0xFFFFu;
    const int l0 = 16 * wave + (mine ? __builtin_ctz(mine) : 0);
    if (MX) {   // without conditions, so that later waits can count these loads; 16 tokens that no row sees: any others
      const int64_t row0 = mine ? __builtin_amdgcn_readlane(at, l0) - (l0 & 15) : 0;
      const uint32_t block = (uint32_t)mx_byte;
      Codes& x = ahead[to];
      x.k[0] = *reinterpret_cast<const uint4*>(a.c.k + row0 * (D / 2) + block * 16);
      x.v[0] = *reinterpret_cast<const uint4*>(a.c.v + row0 * (D / 2) + block * 16);
      x.ks = reinterpret_cast<const uint32_t*>(a.c.ks + row0 * (D / 32))[block / 4];
      x.vs = reinterpret_cast<const uint32_t*>(a.c.vs + row0 * (D / 32))[block / 4];
    } else if (F8) {   // likewise
      const int64_t row0 = mine ? __builtin_amdgcn_readlane(at, l0) - (l0 & 15) : 0;
      const uint8_t *kp = a.c.k + row0 * D, *vp = a.c.v + row0 * D;
      Codes& x = ahead[to];
#pragma unroll
      for (int i = 0; i < kW; ++i) {
        const uint32_t place = (uint32_t)(f8_token(lane) * D + 16 * (lane & 3));
        x.k[i] = *reinterpret_cast<const uint4*>(kp + place + 64 * i);
        x.v[i] = *reinterpret_cast<const uint4*>(vp + place + 64 * i);
      }
      x.ks = a.c.ks[row0 / kF8Block], x.vs = a.c.vs[row0 / kF8Block];
    } else if (mine) {
      const int64_t row0 = __builtin_amdgcn_readlane(at, l0) - (l0 & 15);
      const uint8_t *kp = a.c.k + row0 * (D * 2), *vp = a.c.v + row0 * (D * 2);
#pragma unroll
      for (int i = 0; i < kI; ++i)
        if (mine == 0xFFFFu || ((mine >> (i * kRowsLoad + lane / kC)) & 1)) {
          lds_load16(&lds[to][0][wave * 16 * kC + i * 64], kp, off[i]);
          lds_load16(&lds[to][1][wave * 16 * kC + i * 64], vp, off[i]);
        }
    }
  };
  // Keys that no row sees are masked; their values meet a weight of zero and must be finite.  MXFP4: zeros go to LDS.
  // bf16: what load() leaves out keeps its place there, so the stages start as zeros, and only tokens that some row
  // sees come after.
  auto store = [&](int stage, unsigned long long live) {
    if (MX && lane >> 4 < D / 32) {
      const int row = 16 * wave + mx_row, c0 = 4 * mx_block;
      const Codes& x = ahead[stage];
      const bool dead = !((live >> row) & 1);
      const int at = 8 * (mx_byte & 3);
      const uint32_t ks = dead ? 0 : x.ks >> at & 0xFF, vs = dead ? 0 : x.vs >> at & 0xFF;
      const uint32_t kw[4] = {x.k[0].x, x.k[0].y, x.k[0].z, x.k[0].w}, vw[4] = {x.v[0].x, x.v[0].y, x.v[0].z, x.v[0].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {   // zero codes times 2^-127
        lds[stage][0][kv_chunk<D>(row, c0 + e)] = mx_bf16x8(dead ? 0 : kw[e], ks);
        lds[stage][1][kv_chunk<D>(row, c0 + e)] = mx_bf16x8(dead ? 0 : vw[e], vs);
      }
    }
    if (F8) {
      const Codes& x = ahead[stage];
      // without selects where all 16 tokens are there, as most are
      const bool whole = ((live >> (16 * wave)) & 0xFFFF) == 0xFFFF;
#pragma unroll
      for (int i = 0; i < kW; ++i) {
        const int row = 16 * wave + f8_token(lane), c0 = 8 * i + 2 * (lane & 3);
        uint32_t ks = x.ks, vs = x.vs;
        uint4 k = x.k[i], v = x.v[i];
        if (!whole && !((live >> row) & 1)) ks = vs = 127, k = v = make_uint4(0, 0, 0, 0);
        lds[stage][0][kv_chunk<D>(row, c0)] = f8_bf16x8(make_uint2(k.x, k.y), ks);
        lds[stage][0][kv_chunk<D>(row, c0 + 1)] = f8_bf16x8(make_uint2(k.z, k.w), ks);
        lds[stage][1][kv_chunk<D>(row, c0)] = f8_bf16x8(make_uint2(v.x, v.y), vs);
        lds[stage][1][kv_chunk<D>(row, c0 + 1)] = f8_bf16x8(make_uint2(v.z, v.w), vs);
      }
    }
  };
  if (!CODES) {
    for (int i = tid; i < kT * kC; i += 256) lds[0][1][i] = lds[1][1][i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  // Places of this lane's reads in a tile.  The exchange of chunks follows the token's last four bits, so 16 or 32
  // tokens further on is a constant away.
  int k_at[D / 16], v_at[kDT][2];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) k_at[i] = 16 * kv_chunk<D>(lane & 31, 2 * i + half);
#pragma unroll
  for (int d = 0; d < kDT; ++d)
#pragma unroll
    for (int u = 0; u < 2; ++u)
      v_at[d][u] = 16 * kv_chunk<D>(8 * u + 4 * half + ((lane & 15) >> 2), 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) +
                   8 * (lane & 1);

  // Tiles and pages of a tile on their way while one is worked on.  Codes: tile ti is in ahead[] and in LDS at the
  // parity of ti - first.
  constexpr int kAhead = MX ? 2 : 1;
  unsigned long long live[kAhead + 1] = {};   // of this tile and the next ones, token by token: whether it is there
  int next = 0;
  const bool any = first < end && a.c.pages > 0;
  if (any) {
    int page[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) page[i] = page_of(first + i);
    next = page_of(first + kAhead);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int at = row_of(page[i], first + i);
      live[i] = __ballot(at >= 0);
      load(at, i);
    }
    store(0, live[0]);
  }
  // the queries, here and once: the loop's own waits would count the tiles' loads among theirs
#pragma unroll
  for (int i = 0; i < D / 16; ++i) asm volatile("" : "+v"(qf[i]));
  if (!CODES) lds_load_wait();
  __syncthreads();
  auto step = [&](int ti, auto stage_c) {
    constexpr int stage = decltype(stage_c)::value;
    const int ts = kv_tile_start(span, t0, ti, kT);
    const int at = row_of(next, ti + kAhead);
    live[kAhead] = __ballot(at >= 0);
    next = page_of(ti + kAhead + 1);
    load(at, kAhead == 2 ? stage : stage ^ 1);
    if (ts <= w_hi && live[0] != 0) {
      const char *sk = reinterpret_cast<const char*>(lds[stage][0]), *sv = reinterpret_cast<const char*>(lds[stage][1]);
      v16f s[2] = {};
      v8bf kf[2][D / 16];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < D / 16; ++i) kf[mt][i] = *reinterpret_cast<const v8bf*>(sk + k_at[i] + mt * 32 * kC * 16);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
          s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[mt][i], qf[i], s[mt], 0, 0, 0);
      // four keys ahead of the product that takes them
      __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, 4, 0);
#pragma unroll
      for (int i = 0; i < D / 8 - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 4, 0);
      // unless every row of the wavefront sees every token
      if (live[0] != ~0ull || ts + kT - 1 > w_lo || (w_hi - ts >= a.window && ts + kT > a.sinks)) {
        const unsigned long long see = row_sees(live[0], p, ts + 4 * half, 4 * half, a.window, a.sinks);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const uint32_t bits = (uint32_t)(see >> (32 * mt));
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[mt][i] = bits & (1u << (8 * (i >> 2) + (i & 3))) ? s[mt][i] : -__builtin_inff();
        }
      }
      float tops[4] = {s[0][0], s[0][1], s[1][0], s[1][1]};
#pragma unroll
      for (int i = 2; i < 16; i += 4)
#pragma unroll
        for (int k = 0; k < 4; ++k) {   // v_maximum3
          const v16f& x = s[k >> 1];
          const int at0 = i + 2 * (k & 1);
          if (at0 < 16) tops[k] = attn_max(attn_max(tops[k], x[at0]), x[at0 + 1]);
        }
      float top = attn_max(attn_max(tops[0], tops[1]), attn_max(tops[2], tops[3]));
      top = attn_max(top, __shfl_xor(top, 32));
      if (__any((top - m) * a.scale > kMaxStep)) {
        top = attn_max(top, m);
        const float alpha = __builtin_amdgcn_exp2f((m - top) * a.scale);
        m = top;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < kDT; ++d) o[d] *= alpha;
      }
      const float shift = attn_shift(m, a.scale);
      v8bf pf[4];
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[st >> 1][8 * (st & 1) + i], a.scale, -shift));
          l += e[i];
        }
        pf[st] = __builtin_bit_cast(v8bf, make_uint4(bf16x2(e[0], e[1]), bf16x2(e[2], e[3]), bf16x2(e[4], e[5]),
                                                     bf16x2(e[6], e[7])));
      }
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
          const v8bf vf = join_bf(lds_read_tr(sv + v_at[d][0] + st * 16 * kC * 16), lds_read_tr(sv + v_at[d][1] + st * 16 * kC * 16));
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[st], o[d], 0, 0, 0);
        }
    }
    store(stage ^ 1, live[1]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) live[i] = live[i + 1];
    if (!CODES) lds_load_wait();
    __syncthreads();
  };
  if (any)
    for (int ti = first; ti < end; ti += 2) {   // (codes: in pairs, so that waits stay counted; past the end are no tokens)
      step(ti, std::integral_constant<int, 0>{});
      if (CODES || ti + 1 < end) step(ti + 1, std::integral_constant<int, 1>{});
    }
  l += __shfl_xor(l, 32);
  const int mine = rows - wave * 32 < 32 ? rows - wave * 32 : 32;   // rows of this wavefront
  if (mine <= 0) return;
  // A lane has four neighbouring values of its row at a time; through this wavefront's own quarter of LDS (the tiles
  // are done with) they leave as whole rows.  Chunks are exchanged by row, so that 32 rows at one chunk use all banks.
  const int64_t item = (int64_t)row_g * a.q_heads + qh;
  char* const mem = reinterpret_cast<char*>(&lds[0][0][0]) + wave * (32 * D * 4);
  if (a.slots) {
    const int64_t slot = (int64_t)(first_slot + chunk) * a.b.rows * a.q_heads + item;
    if (half == 0 && lane < mine) a.ml[slot] = make_float2(m, l);
    constexpr int kR = D / 4;   // 16-byte chunks of a row
#pragma unroll
    for (int d = 0; d < kDT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(mem + 16 * ((lane & 31) * kR + ((8 * d + 2 * i + half) ^ (lane & (kR - 1) & 31)))) =
            make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
    wave_sync();
#pragma unroll
    for (int k = 0; k < kR / 2; ++k) {
      const int row = k * (64 / kR) + lane / kR, ch = lane % kR;
      const int64_t to = shfl64(slot, row);
      const float4 x = *reinterpret_cast<const float4*>(mem + 16 * (row * kR + (ch ^ (row & (kR - 1)))));
      if (row < mine) *reinterpret_cast<float4*>(a.po + to * D + 4 * ch) = x;
    }
    return;
  }
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  const int64_t out = (int64_t)row_g * a.ldo + (int64_t)qh * D;
#pragma unroll
  for (int d = 0; d < kDT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(mem + 16 * ((lane & 31) * kC + ((4 * d + i) ^ (lane & (kC - 1)))) + 8 * half) =
          make_uint2(bf16x2(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), bf16x2(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
  wave_sync();
#pragma unroll
  for (int k = 0; k < kC / 2; ++k) {
    const int row = k * (64 / kC) + lane / kC, ch = lane % kC;
    const int64_t to = shfl64(out, row);
    const uint4 x = *reinterpret_cast<const uint4*>(mem + 16 * (row * kC + (ch ^ (row & (kC - 1)))));
    if (row < mine) *reinterpret_cast<uint4*>(a.o + to + 8 * ch) = x;
  }
  if (a.lse && half == 0 && lane < mine) a.lse[item] = attn_lse(m, l, a.scale);
}

}  // namespace sharq
