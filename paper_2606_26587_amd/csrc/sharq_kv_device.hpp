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

// Exponent of the scale of an E4M3 block whose largest magnitude has bits
// `peak`: floor(log2 peak) - 8, or ceil(log2(peak / 448)), which is one more
// where the mantissa is above 1.75 (448 = 1.75 * 2^8), i.e. where adding
// 0x1FFFFF carries.  At least -117: the least code, 2^-9, is then a normal bf16.
// At most 120, of the largest fp32.
constexpr int kF8Least = -117, kF8Most = 120;
constexpr uint32_t kF8Floor = 0u, kF8Ceil = 0x1FFFFFu;
__device__ __forceinline__ int f8_exponent(uint32_t peak, uint32_t rule_bias) {
  const int e = (int)((peak + rule_bias) >> 23) - 135;
  return e < kF8Least ? kF8Least : e;
}

// A value over its block's scale, as it goes to the conversion: saturating at
// the largest code, NaN if it is no finite number.
__device__ __forceinline__ float f8_clamp(float x) {
  const float y = __builtin_fminf(__builtin_fmaxf(x, -448.0f), 448.0f);
  return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : y;
}

// Four fp32 values times 2^-e (as `inv`) -> four E4M3 codes, to nearest even.
__device__ __forceinline__ uint32_t f8_encode4(const float* x, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(f8_clamp(x[0] * inv), f8_clamp(x[1] * inv), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f8_clamp(x[2] * inv), f8_clamp(x[3] * inv), w, true);
}

// Four codes times f, a power of two of at most 1, rounded to E4M3 again.
__device__ __forceinline__ uint32_t f8_rescale4(uint32_t codes, float f) {
  const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, w, true);
}

// Byte SEL (two E2M1 codes) of `codes` under E8M0 scale code e (as the float
// with that exponent field) -> two bf16; every E2M1 value times 2^e is a bf16.
template <int SEL>
__device__ __forceinline__ uint32_t mx_bf16x2(uint32_t codes, float e) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, e, SEL));
}

// Half SEL of `codes` (two E4M3 codes) under the scale with the exponent of e -> two bf16; scales are at least 2^-117,
// so every value is a normal bf16.
template <int SEL>
__device__ __forceinline__ uint32_t f8_bf16x2(uint32_t codes, float e) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, e, SEL != 0));
}

// Eight E4M3 codes -> eight bf16
__device__ __forceinline__ uint4 f8_bf16x8(uint2 codes, uint32_t scale) {
  const float e = __uint_as_float(scale << 23);
  return make_uint4(f8_bf16x2<0>(codes.x, e), f8_bf16x2<1>(codes.x, e), f8_bf16x2<0>(codes.y, e),
                    f8_bf16x2<1>(codes.y, e));
}

// One dword of codes -> eight bf16
__device__ __forceinline__ uint4 mx_bf16x8(uint32_t codes, uint32_t scale) {
  const float e = __uint_as_float(scale << 23);
  return make_uint4(mx_bf16x2<0>(codes, e), mx_bf16x2<1>(codes, e), mx_bf16x2<2>(codes, e), mx_bf16x2<3>(codes, e));
}

}  // namespace sharq
