// Beam search's choice: of the candidates (b, v) of a group's beams and the
// vocabulary, the `beams` best by score_b + x_bv - lse_b, lse_b = ln sum_v e^x_bv.
//
// The logits are read once (k_beam_scan): within a beam the order is the
// logits' own, so the best of a part of a row are found before the row's sum is
// known, and the sum of exponentials is formed beside them with a running
// reference, which moves only when a logit passes it by 8.  What is left, a few
// candidates a part of a row, is joined by one workgroup a group (k_beam_pick).
//
// Measured, bf16: 32 groups of 8 beams over 152064 tokens (78 MB, some beams done)
// 23 us and 7.8 for the join, 3.4 TB/s; one group of 4 over 128256 6.8 and 5.5.
// No one unit bounds the first: vector units are active for 27700 cycles of each
// SIMD (11.5 us at 2.4 GHz; 370 instructions a wavefront and turn, its beginning and
// end among them), a wavefront waits for memory or the others in 43% of its 30000
// cycles and for its turn to issue in 25%, and launch, first loads, five turns and
// the end of 1024 workgroups, all there at once, follow one another.  The second and
// the join are chains of latencies.  One group of 16, 24 and 32 beams over 152064,
// whole calls: 22, 43 and 61 us (3, 5 and 10 turns on 112, 96 and 64 workgroups,
// as the join's LDS allows).  fp32: 16 x 8 x 152064, the same bytes, 27 us for 31.
// Listing single logits during the walk, not a lane's 32 by their largest, took
// 27.6 us; loading a row's last logits one by one, and loads that wait before the
// turn they are for, 36; joining lists with 64-bit exponentials 9 for 5.5.
//
// Candidates of different beams lie close: sums of more than a turn, the
// logarithm and the candidates' keys are held in 64 bits.  All orders are total
// (value, then the lower index), and elements are dealt to threads by their
// column alone, so equal rows give equal sums and the results are a fixed
// function of the inputs.

#include "sharq_attn.hpp"
#include "sharq_serve.hpp"

namespace sharq {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kRefStep = 8.0f;
constexpr float kRefFast = 1000.0f;   // z below 2^-16: its third power is nothing in 64 bits
constexpr int kListCap = 256;   // entries of a wavefront's list
constexpr int kListCut = 64;    // logits beyond which only the best of them stay (at 192: masked 32 x 8 x 152064 63 us, not 46)

// An order of whole numbers that is the floats'; -0 counts as 0.
__device__ __forceinline__ uint32_t order32(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value32(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t order64(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);
  return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double value64(uint64_t k) {
  return __builtin_bit_cast(double, k >> 63 ? k ^ 0x8000000000000000ull : ~k);
}

// 16 bytes of logits, at any element's address.
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef v4u v4u_any __attribute__((aligned(2)));

template <typename T>
__device__ __forceinline__ float as_float(T x) { return (float)x; }

// Logit i of 16 bytes.
template <typename T>
__device__ __forceinline__ float logit(v4u w, int i) {
  if (sizeof(T) == 4) return __uint_as_float(w[i]);
  const uint32_t x = w[i / 2];
  if (__is_same(T, __bf16)) return i % 2 ? bf16_hi(x) : bf16_lo(x);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(i % 2 ? x >> 16 : x));
}

// The `most` best of list[0..n) to out, best first; by one wavefront.  All entries differ.
__device__ __forceinline__ void best_of(const uint64_t* list, int n, int most, uint64_t* out) {
  for (int i = (int)threadIdx.x & 63; i < n; i += 64) {
    const uint64_t x = list[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += list[j] > x;
    if (rank < most) out[rank] = x;
  }
}

// The largest of a wavefront's values (NaN does not count), the same in every lane: by data-parallel moves, which take a
// tenth of the time of six exchanges through LDS.
template <int CTRL>
__device__ __forceinline__ float max_moved(float x) {
  const int o = __builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, 0xF, 0xF, false);
  return __builtin_fmaxf(x, __int_as_float(o));
}
__device__ __forceinline__ float wave_max(float x) {
  x = max_moved<0x111>(x);   // rows of 16: shifted by 1, 2, 4, 8
  x = max_moved<0x112>(x);
  x = max_moved<0x114>(x);
  x = max_moved<0x118>(x);
  x = max_moved<0x142>(x);   // the last of a row to the next, of the first half to the second
  x = max_moved<0x143>(x);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Their sum in the last lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ double sum_moved(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, false);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) {
  x = sum_moved<0x111, 0xF>(x);
  x = sum_moved<0x112, 0xF>(x);
  x = sum_moved<0x114, 0xF>(x);
  x = sum_moved<0x118, 0xF>(x);
  x = sum_moved<0x142, 0xA>(x);   // into rows 1 and 3
  return sum_moved<0x143, 0xC>(x);   // into rows 2 and 3
}

// x times 2^e, e a whole number of any size (not above 0).
__device__ __forceinline__ double times_exp2(double x, double e) {
  return __builtin_amdgcn_ldexp(x, e > -4000.0 ? (int)e : -4000);
}

// The whole exponent of a reference, and what is left of it (a reference past 2^53 has nothing left).
__device__ __forceinline__ double exponent_of(float ref, float& rest) {
  const double y = (double)ref * 1.44269504088896341, e = __builtin_rint(y);
  rest = (float)(y - e);
  return e;
}

// An entry of a sorted list: the value's order above, the complement of its column below, so that of equal values the
// lower column is the better.
__device__ __forceinline__ uint64_t entry_of(float x, int col) { return (uint64_t)order32(x) << 32 | (uint32_t)~col; }

// The `most`-th largest of n values in LDS (n is at least that), by one wavefront.
__device__ __forceinline__ float least_of(const float* value, int n, int most) {
  float found = -__builtin_inff();
  for (int i = (int)threadIdx.x & 63; i < n; i += 64) {
    const float x = value[i];
    int reach = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) reach += value[j] >= x;
    if (reach >= most) found = __builtin_fmaxf(found, x);
  }
  return wave_max(found);
}

// The same of the wavefront's own values, one a lane.
__device__ __forceinline__ float least_of_lanes(float x, int most) {
  int reach = 0;
#pragma unroll 16
  for (int j = 0; j < 64; ++j) reach += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), j)) >= x;
  return wave_max(reach >= most ? x : -__builtin_inff());
}

// A part of a row: workgroup (row, chunk), whose wavefronts work apart, each on its 2048 of a turn's 8192 logits.  During
// the walk only a lane's largest of a turn is looked at: its 32 logits are listed where that may still be chosen.  The
// `beams`-th largest of such maxima is a bound (so many logits reach it), and at the end the few turns of a lane whose
// maximum reaches the last bound, about `beams` of them, are read once more.
template <typename T>
__global__ __launch_bounds__(256) void k_beam_scan(BeamArgs a) {
  constexpr int kVec = 16 / (int)sizeof(T), kLoads = kBeamPer / kVec;
  __shared__ uint64_t lds_entry[4][kListCap], lds_best[4][kMaxBeams];
  __shared__ float lds_value[4][kListCap];
  __shared__ int lds_turn[4][kListCap];
  __shared__ float lds_least[4];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row = (int)(blockIdx.x / (unsigned)a.chunks), chunk = (int)(blockIdx.x % (unsigned)a.chunks);
  const T* const x = static_cast<const T*>(a.logits) + (int64_t)row * a.ld;
  uint64_t *const entry = lds_entry[wave], *const best = lds_best[wave];
  float* const value = lds_value[wave];    // of a listed turn of a lane: its largest logit, and
  int* const turn = lds_turn[wave];        // its first column
  int n = 0;                         // how many there are
  float least = -__builtin_inff();   // what has to be passed: `beams` logits before reach it
  float ref = -__builtin_inff();
  float rest = 0.0f;
  double sum = 0.0, exponent = -__builtin_inf();
  v4u w[kLoads];   // a turn's logits, on their way during the turn before
  const bool some = a.vocab >= kVec;
  auto load = [&](int base) {   // where the row has ended: others of it
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int at = base + (k * 64 + lane) * kVec;
      w[k] = *reinterpret_cast<const v4u_any*>(x + (at + kVec <= a.vocab ? at : 0));
    }
  };
  auto keep = [&](int limit) {   // of the list what reaches `least`; what equals it before column `limit` only
    int kept = 0;
    for (int i = 0; i < n; i += 64) {
      const float y = i + lane < n ? value[i + lane] : -__builtin_inff();
      const int t = i + lane < n ? turn[i + lane] : 0;
      const unsigned long long who = __ballot(i + lane < n && y >= least && (y > least || t < limit));
      wave_sync();
      if ((who >> lane) & 1) {
        const int to = kept + __popcll(who & ((1ull << lane) - 1));
        value[to] = y, turn[to] = t;
      }
      kept += __popcll(who);
    }
    n = kept;
    wave_sync();
  };
  const int end = (chunk + 1) * a.tiles * kBeamTile < a.vocab ? (chunk + 1) * a.tiles * kBeamTile : a.vocab;
  const int begin = chunk * a.tiles * kBeamTile + wave * (64 * kBeamPer);
  if (begin < end && some) load(begin);
  if (a.done && a.done[row]) return;   // its one candidate needs no logits
  for (int base = begin; base < end; base += kBeamTile) {
    float v[kBeamPer];
#pragma unroll
    for (int i = 0; i < kBeamPer; ++i) v[i] = logit<T>(w[i / kVec], i % kVec);
    if (base + 64 * kBeamPer > a.vocab) {   // the row ends in this turn, perhaps inside of 16 bytes
      const int over = a.vocab % kVec, whole = a.vocab - over;
      const float mine = lane < over ? as_float(x[whole + lane]) : -__builtin_inff();
#pragma unroll
      for (int i = 0; i < kBeamPer; ++i) {
        const int at = base + (i / kVec * 64 + lane) * kVec;
        const float o = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), i % kVec));
        v[i] = at < whole ? v[i] : at == whole ? o : -__builtin_inff();
      }
    }
    if (base + kBeamTile < end && some) load(base + kBeamTile);
    float top = v[0];
#pragma unroll
    for (int i = 1; i < kBeamPer; ++i) top = __builtin_fmaxf(top, v[i]);
    const float all = wave_max(top);
    // Terms are 2^((x - ref) log2 e + rest) = e^x 2^-exponent, with a whole exponent: sums move from one to another exactly.
    if (all > ref + kRefStep || (ref == -__builtin_inff() && all > ref)) {
      const double e = exponent_of(all, rest);
      sum = times_exp2(sum, exponent - e);   // 0 of the first reference's
      ref = all, exponent = e;
    }
    if (ref != -__builtin_inff()) {
      float s[8] = {};
      double part = 1.0;
      if (__builtin_fabsf(ref) < kRefFast) {
        // x log2 e - exponent in one step.  The constant's error counts for x, not x - ref: ref's part of it, z, is taken
        // out of the sum.
        const float e = -(float)exponent;
#pragma unroll
        for (int i = 0; i < kBeamPer; ++i) s[i & 7] += __builtin_amdgcn_exp2f(__builtin_fmaf(v[i], kLog2e, e));
        const double z = (double)ref * ((1.44269504088896341 - (double)kLog2e) * 0.69314718055994531);
        part = 1.0 + z * (1.0 + 0.5 * z);
      } else {
#pragma unroll
        for (int i = 0; i < kBeamPer; ++i) s[i & 7] += __builtin_amdgcn_exp2f(__builtin_fmaf(v[i] - ref, kLog2e, rest));
      }
      sum += part * (double)(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
    } else {   // nothing yet, unless it is a NaN
#pragma unroll
      for (int i = 0; i < kBeamPer; ++i)
        if (v[i] != v[i]) sum = __builtin_nan("");
    }
    unsigned long long who = __ballot(top > least);
    if (__popcll(who) > (n == 0 ? a.beams : 2 * a.beams)) {
      const float bound = least_of_lanes(top, a.beams);
      if (bound > least) least = bound, who = __ballot(top >= least);
    }
    if (who) {
      if ((who >> lane) & 1) {
        const int to = n + __popcll(who & ((1ull << lane) - 1));
        value[to] = top, turn[to] = base + lane * kVec;
      }
      n += __popcll(who);
      if (n > kListCap - 64) {
        wave_sync();
        least = __builtin_fmaxf(least, least_of(value, n, a.beams));
        keep(a.vocab);
        // Many equal ones are left.  The list is in the order of turns: what equals the bound behind the turn that has
        // the `beams`-th is not chosen, so there are at most 63 more of this turn, and fewer than `beams` above.
        if (n > kListCap - 64) {
          const int reached = __builtin_amdgcn_readfirstlane(turn[a.beams - 1]) - begin;
          keep(begin + (reached / kBeamTile + 1) * kBeamTile);
        }
      }
    }
  }
  sum = wave_sum(sum);
  const int64_t part = (int64_t)row * a.chunks + chunk;
  if (lane == 63) a.parts[part * 4 + wave] = BeamPart{sum, ref, 0};
  // What one wavefront's logits say holds for all four.
  wave_sync();
  if (n >= a.beams) least = __builtin_fmaxf(least, least_of(value, n, a.beams));
  if (lane == 0) lds_least[wave] = least;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) least = __builtin_fmaxf(least, lds_least[i]);
  keep(a.vocab);
  int found = 0;
  {
    // Two turns of a lane at a time, four such loads on their way.  Where many logits reach the bound (a mask's, wide
    // beams) the best so far take their places, and what is not better than the last of these stays out.  A part of a row
    // with fewer than `beams` tokens left by a mask of the type's lowest value: 2048 equal logits.  10 tokens left of
    // 152064, 32 x 8 beams 46 us (unmasked 31), 1 x 32 43 us (53); walking the part once for each beam took 486 and 1513.
    const int k = lane % kBeamPer, off = k / kVec * 64 * kVec + k % kVec;
    uint64_t floor = 0;
    for (int first = 0; first < n; first += 8) {
      float y[4];
      int col[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = first + 2 * j + lane / kBeamPer;
        col[j] = i < n ? turn[i] + off : a.vocab;
        y[j] = col[j] < a.vocab ? as_float(x[col[j]]) : -__builtin_inff();
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t e = entry_of(y[j], col[j]);
        const unsigned long long who = __ballot(y[j] >= least && y[j] > -__builtin_inff() && e > floor);
        if ((who >> lane) & 1) entry[found + __popcll(who & ((1ull << lane) - 1))] = e;
        found += __popcll(who);
        if (found > kListCut) {
          wave_sync();
          best_of(entry, found, a.beams, best);
          wave_sync();
          found = a.beams;
          if (lane < found) entry[lane] = best[lane];
          floor = best[found - 1];
          wave_sync();
        }
      }
    }
    wave_sync();
    best_of(entry, found, a.beams, best);
    found = found < a.beams ? found : a.beams;
  }
  if (lane >= found && lane < a.beams) best[lane] = 0;
  __syncthreads();
  if (wave != 0) return;
  // the four lists' best; entries of 0 are none
  n = 0;
  for (int i = 0; i < 4 * a.beams; i += 64) {
    const int at = i + lane;
    const uint64_t e = at < 4 * a.beams ? lds_best[at / a.beams][at % a.beams] : 0;
    const unsigned long long is = __ballot(e != 0);
    if (e) entry[n + __popcll(is & ((1ull << lane) - 1))] = e;
    n += __popcll(is);
  }
  wave_sync();
  uint64_t* const out = a.lists + part * a.beams;
  best_of(entry, n, a.beams, out);
  for (int i = n + lane; i < a.beams; i += 64) out[i] = 0;
}

struct __attribute__((aligned(16))) BeamKey {
  uint64_t order;     // of the score, 0: none
  uint32_t at, own;   // beam * vocab + token; the logit's order
};
// Of equal scores the lower beam's is the better.  Within a beam the logits decide: under a score of large magnitude
// different ones may give the same sum.
__device__ __forceinline__ bool better_equal(const BeamKey& x, const BeamKey& y, uint32_t vocab) {
  if (x.own == y.own || x.at / vocab != y.at / vocab) return x.at < y.at;
  return x.own > y.own;
}

// At least kBeamLists; a wavefront a beam forms the sums (32 groups of 8: half a microsecond less than with 256 threads).
constexpr int kPickThreads = 512;

// Joins a group's lists.  A thread has one list, whose entries come best first.  As `beams` lists reach the `beams`-th of
// a wavefront's first entries, nothing below can be chosen; what is not below it is ranked.
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(BeamArgs a) {
  extern __shared__ BeamKey found[];   // up to as many as there are entries
  __shared__ double base_of[kMaxBeams], lse_of[kMaxBeams];
  __shared__ uint8_t done_of[kMaxBeams];
  __shared__ BeamPart part_of[kBeamLists];
  __shared__ uint32_t bound_of[kPickThreads / 64];
  __shared__ int count;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), beams = a.beams;
  const int lists = beams * a.chunks, entries = lists * beams;
  uint64_t* const entry = reinterpret_cast<uint64_t*>(found + entries);   // [lists][beams]
  const int64_t row0 = (int64_t)blockIdx.x * beams;
  const uint64_t* const from = a.lists + row0 * a.chunks * beams;
  const int b = tid < lists ? tid / a.chunks : 0;
  BeamPart q[4] = {};
  if (tid < lists) {   // all loads on their way together (a beam that is done left its own unwritten)
    const BeamPart* const p = a.parts + (row0 * a.chunks + tid) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = p[i];
  }
  uint8_t done = 0;
  float score = 0.0f;
  if (tid < beams) {
    if (a.done) done = a.done[row0 + tid];
    score = a.scores[row0 + tid];
  }
  for (int i = tid; i < entries; i += kPickThreads) entry[i] = from[i];
  if (tid == 0) count = 0;
  if (tid < beams) done_of[tid] = done != 0, base_of[tid] = (double)score;
  // a thread's four parts of a sum, then a wavefront a beam
  {
    const float top = __builtin_fmaxf(__builtin_fmaxf(q[0].ref, q[1].ref), __builtin_fmaxf(q[2].ref, q[3].ref));
    float rest;
    const double exponent = exponent_of(top, rest);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (q[i].sum != 0.0) sum += times_exp2(q[i].sum, exponent_of(q[i].ref, rest) - exponent);
    if (tid < lists) part_of[tid] = BeamPart{sum, top, 0};
  }
  __syncthreads();
  for (int i = wave; i < beams; i += kPickThreads / 64) {
    BeamPart p{0.0, -__builtin_inff(), 0};
    for (int c = lane; c < a.chunks; c += 64) {   // more than 64 where the beams are few
      const BeamPart o = part_of[i * a.chunks + c];
      float rest;
      const float top = __builtin_fmaxf(p.ref, o.ref);
      const double e = exponent_of(top, rest);
      double sum = o.sum != 0.0 ? times_exp2(o.sum, exponent_of(o.ref, rest) - e) : 0.0;
      if (p.sum != 0.0) sum += times_exp2(p.sum, exponent_of(p.ref, rest) - e);
      p = BeamPart{sum, top, 0};
    }
    float rest, left;
    const float top = wave_max(p.ref);
    const double e = exponent_of(top, left);
    const double sum = wave_sum(p.sum != 0.0 ? times_exp2(p.sum, exponent_of(p.ref, rest) - e) : 0.0);
    // no logit: -inf, and no candidate
    if (lane == 63) lse_of[i] = (double)top + (log2(sum) - (double)left) * 0.69314718055994530942;
  }
  __syncthreads();
  auto key_of = [&](int b, uint64_t e) {
    BeamKey k{0, 0, 0};
    double total;
    if (done_of[b]) {
      total = base_of[b], k.at = (uint32_t)(b * a.vocab + a.eos);
    } else {
      if (e == 0) return k;
      total = base_of[b] + ((double)value32((uint32_t)(e >> 32)) - lse_of[b]);
      k.at = (uint32_t)(b * a.vocab) + (uint32_t)~(uint32_t)e, k.own = (uint32_t)(e >> 32);
    }
    if (total > -__builtin_inf() && total < __builtin_inf()) k.order = order64(total);
    return k;
  };
  const bool mine = tid < lists && (!done_of[b] || tid % a.chunks == 0);
  BeamKey head{0, 0, 0};
  if (mine) head = key_of(b, entry[tid * beams]);
  // The upper halves of the orders will do: the largest one that `beams` first entries reach.
  const uint32_t upper = (uint32_t)(head.order >> 32);
  int reach = 0;
#pragma unroll 8
  for (int j = 0; j < 64; ++j) reach += (uint32_t)__builtin_amdgcn_readlane((int)upper, j) >= upper;
  uint32_t bound = reach >= beams ? upper : 0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)bound, d);
    bound = o > bound ? o : bound;
  }
  if (lane == 0) bound_of[wave] = bound;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPickThreads / 64; ++w) bound = bound_of[w] > bound ? bound_of[w] : bound;
  if (mine) {
    BeamKey k = head;
    for (int i = 0; k.order != 0 && (uint32_t)(k.order >> 32) >= bound;) {
      found[atomicAdd(&count, 1)] = k;   // in any order: they are ranked below
      if (++i == beams || done_of[b]) break;
      k = key_of(b, entry[tid * beams + i]);
    }
  }
  __syncthreads();
  const int n = count;
  for (int i = tid; i < n; i += kPickThreads) {
    const BeamKey k = found[i];
    int r = 0, same = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) r += found[j].order > k.order, same += found[j].order == k.order;
    if (same > 1)
      for (int j = 0; j < n; ++j)
        if (found[j].order == k.order) r += better_equal(found[j], k, (uint32_t)a.vocab);
    if (r >= beams) continue;
    const int parent = (int)(k.at / (uint32_t)a.vocab), token = (int)(k.at % (uint32_t)a.vocab);
    a.scores_out[row0 + r] = (float)value64(k.order);
    a.parents[row0 + r] = parent;
    a.tokens[row0 + r] = token;
    if (a.done_out) a.done_out[row0 + r] = done_of[parent] || token == a.eos;
  }
  for (int r = n + tid; r < beams; r += kPickThreads) {   // no candidate left
    a.scores_out[row0 + r] = -__builtin_inff();
    a.parents[row0 + r] = r;
    a.tokens[row0 + r] = -1;
    if (a.done_out) a.done_out[row0 + r] = done_of[r];
  }
}

hipError_t launch_beam_select(const BeamArgs& a, int64_t groups, int dtype, hipStream_t st) {
  const dim3 g((unsigned)(groups * a.beams * a.chunks));
  if (dtype == 0) k_beam_scan<__bf16><<<g, 256, 0, st>>>(a);
  else if (dtype == 1) k_beam_scan<_Float16><<<g, 256, 0, st>>>(a);
  else k_beam_scan<float><<<g, 256, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t lds = (size_t)beam_lds(a.beams, a.chunks);
  k_beam_pick<<<(unsigned)groups, kPickThreads, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace sharq
