// Beam search's choice: of the candidates (b, v) of a group's beams and the
// vocabulary, the `beams` best by score_b + x_bv - lse_b, lse_b = ln sum_v e^x_bv.
//
// The logits are read once (k_beam_scan): within a beam the order is the
// logits' own, so the best of a part of a row are found before the row's sum is
// known, and the sum of exponentials is formed beside them with a running
// reference, which moves only when a logit passes it by 8.  What is left, a few
// candidates a part of a row, is joined by one workgroup a group (k_beam_pick).
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
constexpr int kListCap = 256;   // entries of a wavefront's list, while a turn's candidates join it

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

template <typename T>
__device__ __forceinline__ float as_float(T x) { return (float)x; }

// 16 bytes at any element's address.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
  T v[N];
};

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

__device__ __forceinline__ uint64_t wave_max64(uint64_t x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = (uint64_t)(uint32_t)__shfl_xor((int)(uint32_t)x, d) |
                       (uint64_t)(uint32_t)__shfl_xor((int)(uint32_t)(x >> 32), d) << 32;
    x = o > x ? o : x;
  }
  return x;
}

// A part of a row: workgroup (row, chunk), whose wavefronts work apart, each on its 2048 of a turn's 8192 logits.  An
// entry of a list: the value's order above, the complement of its column below, so that of equal values the lower
// column is the better.
template <typename T>
__global__ __launch_bounds__(256) void k_beam_scan(BeamArgs a) {
  constexpr int kVec = 16 / (int)sizeof(T), kLoads = kBeamPer / kVec;
  __shared__ uint64_t lds_list[4][kListCap], lds_best[4][kMaxBeams];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row = (int)(blockIdx.x / (unsigned)a.chunks), chunk = (int)(blockIdx.x % (unsigned)a.chunks);
  if (a.done && a.done[row]) return;   // its one candidate needs no logits
  const T* const x = static_cast<const T*>(a.logits) + (int64_t)row * a.ld;
  uint64_t *const list = lds_list[wave], *const best = lds_best[wave];
  int have = 0;                      // entries of best[]
  float least = -__builtin_inff();   // what a value has to pass: that of the last of `beams` entries
  float ref = -__builtin_inff();
  double sum = 0.0;
  for (int tile = chunk * a.tiles; tile < (chunk + 1) * a.tiles; ++tile) {
    const int base = tile * kBeamTile + wave * (64 * kBeamPer);
    if (base >= a.vocab) break;
    float v[kBeamPer];
    if (base + 64 * kBeamPer <= a.vocab) {   // all loads on their way together
      Vec<T, kVec> w[kLoads];
#pragma unroll
      for (int k = 0; k < kLoads; ++k) w[k] = *reinterpret_cast<const Vec<T, kVec>*>(x + base + (k * 64 + lane) * kVec);
#pragma unroll
      for (int i = 0; i < kBeamPer; ++i) v[i] = as_float(w[i / kVec].v[i % kVec]);
    } else {
#pragma unroll
      for (int i = 0; i < kBeamPer; ++i) {
        const int at = base + (i / kVec * 64 + lane) * kVec + i % kVec;
        v[i] = at < a.vocab ? as_float(x[at]) : -__builtin_inff();
      }
    }
    float top = v[0];
#pragma unroll
    for (int i = 1; i < kBeamPer; ++i) top = __builtin_fmaxf(top, v[i]);
    float all = top;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) all = __builtin_fmaxf(all, __shfl_xor(all, d));
    if (all > ref + kRefStep || (ref == -__builtin_inff() && all > ref)) {
      sum *= exp2((double)(ref - all) * 1.44269504088896341);   // 0 of the first reference's
      ref = all;
    }
    if (ref != -__builtin_inff()) {
      float s[8] = {};
#pragma unroll
      for (int i = 0; i < kBeamPer; ++i) s[i & 7] += __builtin_amdgcn_exp2f((v[i] - ref) * kLog2e);
      sum += (double)(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
    } else {   // nothing yet, unless it is a NaN
#pragma unroll
      for (int i = 0; i < kBeamPer; ++i)
        if (v[i] != v[i]) sum = __builtin_nan("");
    }
    const unsigned long long above = __ballot(top > least);
    if (above == 0) continue;
    // Where many lanes have something, the `beams`-th of their best is a bound as well: so many values reach it.
    uint32_t bound = order32(least) + 1;
    if (__popcll(above) > a.beams) {
      const uint32_t mine = order32(top);
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < 64; ++j) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)mine, j);
        rank += o > mine || (o == mine && j < lane);
      }
      const int l = __builtin_ctzll(__ballot(rank == a.beams - 1));
      const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)mine, l);
      bound = at > bound ? at : bound;
    }
    wave_sync();
    for (int i = lane; i < have; i += 64) list[i] = best[i];
    int n = have;
#pragma unroll
    for (int i = 0; i < kBeamPer; ++i) {
      const uint32_t o = order32(v[i]);
      const bool in = o >= bound && v[i] == v[i];
      const unsigned long long who = __ballot(in);
      if (who) {
        const int to = n + __popcll(who & ((1ull << lane) - 1));
        const int col = base + (i / kVec * 64 + lane) * kVec + i % kVec;
        if (in && to < kListCap) list[to] = (uint64_t)o << 32 | (uint32_t)~col;
        n += __popcll(who);
      }
    }
    wave_sync();
    if (n <= kListCap) {
      best_of(list, n, a.beams, best);
      have = n < a.beams ? n : a.beams;
    } else {   // more values at the bound than the list holds: one after the other
      uint64_t last = ~0ull;
      const uint64_t old = lane < have ? best[lane] : 0;
      wave_sync();
      for (have = 0; have < a.beams; ++have) {
        uint64_t mine = old < last ? old : 0;
#pragma unroll
        for (int i = 0; i < kBeamPer; ++i) {
          const int col = base + (i / kVec * 64 + lane) * kVec + i % kVec;
          const uint64_t e = (uint64_t)order32(v[i]) << 32 | (uint32_t)~col;
          if (v[i] > -__builtin_inff() && e < last && e > mine) mine = e;
        }
        mine = wave_max64(mine);
        if (mine == 0) break;
        if (lane == 0) best[have] = mine;
        last = mine;
      }
    }
    wave_sync();
    if (have == a.beams) least = value32((uint32_t)(best[have - 1] >> 32));
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t b = __builtin_bit_cast(uint64_t, sum);
    sum += __builtin_bit_cast(double, (uint64_t)(uint32_t)__shfl_xor((int)(uint32_t)b, d) |
                                          (uint64_t)(uint32_t)__shfl_xor((int)(uint32_t)(b >> 32), d) << 32);
  }
  const int64_t part = (int64_t)row * a.chunks + chunk;
  if (lane == 0) a.parts[part * 4 + wave] = BeamPart{sum, ref, 0};
  for (int i = have + lane; i < a.beams; i += 64) best[i] = 0;
  __syncthreads();
  if (wave != 0) return;
  // the four lists' best; entries of 0 are none
  int n = 0;
  for (int i = 0; i < 4 * a.beams; i += 64) {
    const int at = i + lane;
    const uint64_t e = at < 4 * a.beams ? lds_best[at / a.beams][at % a.beams] : 0;
    const unsigned long long is = __ballot(e != 0);
    if (e) list[n + __popcll(is & ((1ull << lane) - 1))] = e;
    n += __popcll(is);
  }
  wave_sync();
  uint64_t* const out = a.lists + part * a.beams;
  best_of(list, n, a.beams, out);
  for (int i = n + lane; i < a.beams; i += 64) out[i] = 0;
}

struct BeamKey {
  uint64_t order;   // of the score, 0: none
  uint32_t at;      // beam * vocab + token
};
__device__ __forceinline__ bool better(const BeamKey& x, const BeamKey& y) {
  return x.order > y.order || (x.order == y.order && x.at < y.at);
}

// Joins a group's lists.  A thread has one list, whose entries come best first: the `beams`-th best of a wavefront's
// first entries bounds what can be chosen, and what reaches the bound is ranked.
__global__ __launch_bounds__(256) void k_beam_pick(BeamArgs a) {
  extern __shared__ uint64_t lds[];
  __shared__ double base_of[kMaxBeams], lse_of[kMaxBeams];
  __shared__ uint8_t done_of[kMaxBeams];
  __shared__ BeamKey bound_of[4];
  __shared__ int count;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, beams = a.beams;
  const int lists = beams * a.chunks, entries = lists * beams;
  uint64_t* const entry = lds;                       // [lists][beams]
  uint64_t* const order = lds + entries;             // of those that reach the bound: their orders, and
  uint32_t* const place = reinterpret_cast<uint32_t*>(order + (lists + 63) / 64 * beams * beams);   // their places
  const int64_t row0 = (int64_t)blockIdx.x * beams;
  const uint64_t* const from = a.lists + row0 * a.chunks * beams;
  for (int i = tid; i < entries; i += 256) entry[i] = from[i];   // a beam that is done left its own unwritten
  if (tid == 0) count = 0;
  for (int b = wave; b < beams; b += 4) {
    const bool done = a.done && a.done[row0 + b];
    float top = -__builtin_inff();
    double sum = 0.0;
    const BeamPart* const parts = a.parts + (row0 + b) * a.chunks * 4;
    if (!done) {
      for (int i = lane; i < a.chunks * 4; i += 64) top = __builtin_fmaxf(top, parts[i].top);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, d));
      for (int i = lane; i < a.chunks * 4; i += 64)
        if (parts[i].sum != 0.0) sum += parts[i].sum * exp((double)parts[i].top - (double)top);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint64_t u = __builtin_bit_cast(uint64_t, sum);
        sum += __builtin_bit_cast(double, (uint64_t)(uint32_t)__shfl_xor((int)(uint32_t)u, d) |
                                              (uint64_t)(uint32_t)__shfl_xor((int)(uint32_t)(u >> 32), d) << 32);
      }
    }
    if (lane == 0) {
      done_of[b] = done;
      base_of[b] = (double)a.scores[row0 + b];
      lse_of[b] = (double)top + log(sum);   // no logit: -inf - inf, and no candidate
    }
  }
  __syncthreads();
  auto key_of = [&](int b, uint64_t e) {
    BeamKey k{0, 0};
    double total;
    if (done_of[b]) {
      total = base_of[b], k.at = (uint32_t)(b * a.vocab + a.eos);
    } else {
      if (e == 0) return k;
      total = base_of[b] + ((double)value32((uint32_t)(e >> 32)) - lse_of[b]);
      k.at = (uint32_t)(b * a.vocab) + (uint32_t)~(uint32_t)e;
    }
    if (total > -__builtin_inf()) k.order = order64(total);
    return k;
  };
  const int b = tid < lists ? tid / a.chunks : 0;
  const bool mine = tid < lists && (!done_of[b] || tid % a.chunks == 0);
  BeamKey head{0, 0};
  if (mine) head = key_of(b, entry[tid * beams]);
  int rank = 0;
  for (int j = 0; j < 64; ++j) {
    const BeamKey o{(uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)head.order, j) |
                        (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(head.order >> 32), j) << 32,
                    (uint32_t)__builtin_amdgcn_readlane((int)head.at, j)};
    rank += better(o, head) || (o.order == head.order && o.at == head.at && j < lane);
  }
  if (rank == beams - 1) bound_of[wave] = head;
  __syncthreads();
  BeamKey bound = bound_of[0];
  for (int w = 1; w < 4; ++w)
    if (better(bound_of[w], bound)) bound = bound_of[w];
  if (mine) {
    BeamKey k = head;
    for (int i = 0; k.order != 0 && !better(bound, k);) {
      const int to = atomicAdd(&count, 1);   // in any order: the places are ranked below
      order[to] = k.order, place[to] = k.at;
      if (++i == beams || done_of[b]) break;
      k = key_of(b, entry[tid * beams + i]);
    }
  }
  __syncthreads();
  const int n = count;
  for (int i = tid; i < n; i += 256) {
    const BeamKey k{order[i], place[i]};
    int r = 0;
    for (int j = 0; j < n; ++j) r += better(BeamKey{order[j], place[j]}, k);
    if (r >= beams) continue;
    const int parent = (int)(k.at / (uint32_t)a.vocab), token = (int)(k.at % (uint32_t)a.vocab);
    a.scores_out[row0 + r] = (float)value64(k.order);
    a.parents[row0 + r] = parent;
    a.tokens[row0 + r] = token;
    if (a.done_out) a.done_out[row0 + r] = done_of[parent] || token == a.eos;
  }
  for (int r = n + tid; r < beams; r += 256) {   // no candidate left
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
  k_beam_pick<<<(unsigned)groups, 256, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace sharq
