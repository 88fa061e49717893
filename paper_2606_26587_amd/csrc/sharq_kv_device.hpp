// Device side of the paged key/value cache: the sequences of a call, and the
// element conversions that the append, the read-back and the attention share.
#pragma once

#include "sharq_device.hpp"
#include "sharq_kv.hpp"

namespace sharq {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// Rows and cached length of sequence s.  The offsets and lengths are device
// data that no call on the host has looked at: clamped, so that whatever they
// hold every index derived from them stays inside its buffer.
struct SeqRows {
  int first, n, len;
};

__device__ __forceinline__ SeqRows seq_rows(const KvBatchArgs& b, int s) {
  SeqRows r;
  r.first = kv_clamp(b.offs[s], 0, b.rows);
  r.n = kv_clamp(b.offs[s + 1], r.first, b.rows) - r.first;
  r.len = kv_clamp(b.lens[s], 0, b.max_len);
  return r;
}

// The sequence that holds `row` (b.seqs: none, a row behind the last one),
// found by a whole wavefront: each round its lanes sample 64 of the remaining
// offsets, so a thousand sequences take two dependent loads.
__device__ __forceinline__ int find_seq(const KvBatchArgs& b, int row) {
  const int lane = (int)(threadIdx.x & 63);
  int lo = 0, hi = b.seqs;   // the number of sequences that end at or before `row` is in [lo, hi]
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) / 64, i = lo + (lane + 1) * step - 1;
    const int c = __popcll(__ballot(i < hi && b.offs[i + 1] <= row));
    lo += c * step;
    hi = hi < lo + step ? hi : lo + step;
  }
  const int i = lo + lane;
  return lo + __popcll(__ballot(i < hi && b.offs[i + 1] <= row));
}

// fp32 pair -> two bf16, to nearest even, the first in the low half
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
  v2bf r;
  r[0] = (__bf16)a;
  r[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, r);
}

// Byte SEL (two E2M1 codes) of `codes` under E8M0 scale code e (as the float
// with that exponent field) -> two bf16; every E2M1 value times 2^e is a bf16.
template <int SEL>
__device__ __forceinline__ uint32_t mx_bf16x2(uint32_t codes, float e) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, e, SEL));
}

// One dword of codes -> eight bf16
__device__ __forceinline__ uint4 mx_bf16x8(uint32_t codes, uint32_t scale) {
  const float e = __uint_as_float(scale << 23);
  return make_uint4(mx_bf16x2<0>(codes, e), mx_bf16x2<1>(codes, e), mx_bf16x2<2>(codes, e), mx_bf16x2<3>(codes, e));
}

}  // namespace sharq
