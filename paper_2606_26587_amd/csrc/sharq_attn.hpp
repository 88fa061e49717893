// What the attention kernels share: their arguments, the layout of a tile of
// keys or values in LDS, and where a workgroup's results go.
#pragma once

#include "sharq_kv_device.hpp"

namespace sharq {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

struct AttnArgs {
  const uint16_t* q;
  int64_t ldq;
  uint16_t* o;
  int64_t ldo;
  float* lse;
  KvBatchArgs b;
  KvCacheArgs c;
  const int32_t* prefix_table;
  int prefix_len;
  int t0;            // a sequence's own part begins at this token: prefix_len, or 0 (the whole sequence)
  int few_rows;      // sequences of up to this many rows to a key/value head are not the many-row kernel's
  int group, q_heads, window, sinks;
  float scale;       // of the scores, times log2 e
  // partial results, where the tokens of a row are split over workgroups: slot
  // s of row r and head h holds the running maximum (of the unscaled scores)
  // and the sum of the softmax, ml[(s * rows + r) * q_heads + h], and the unnormalised
  // output po[same][D], all fp32.  slots 0: results go to o.
  float2* ml;
  float* po;
  int slots;
};

// Position of 16-byte chunk c of token t's row in an LDS tile of D bf16 a row.
// The keys are read 16 tokens at a time at one chunk, the values 4 tokens at 64
// consecutive bytes or 8 at 32: under this exchange of chunks all of them fall
// on all 64 banks.
template <int D>
__device__ __forceinline__ int kv_chunk(int t, int c) {
  constexpr int kC = D / 8;
  const int f = D == 128 ? ((t & 3) << 2 | ((t >> 2) & 1) << 1 | ((t >> 3) & 1))
                         : (((t >> 1) & 1) << 2 | ((t >> 2) & 1) << 1 | ((t >> 3) & 1));
  return t * kC + (c ^ f);
}

// The token of 16 that a lane (of each 16) writes to LDS from an MXFP4 cache:
// 8 lanes in a row, which are written together, reach 8 different 16-byte places
// of 128 bytes under kv_chunk's exchange.
template <int D>
__device__ __forceinline__ int mx_token(int lane) {
  const int l = lane & 15;
  return D == 128 ? (l & 1) | (l & 6) << 1 | (l & 8) >> 2 : (l & 7) << 1 | l >> 3;
}

// The token of 16 whose 16 values from 16 (lane & 3) on (and, of heads of 128, from 64 further on) a lane writes to LDS
// from an E4M3 cache.  8 lanes in a row take two tokens that are 8 apart, which kv_chunk's exchange puts at odd and at
// even places: the first of the two chunks of all 8, and the second, reach 8 different ones of 128 bytes.
__device__ __forceinline__ int f8_token(int lane) { return lane >> 3 | (lane & 4) << 1; }

// Transposing LDS read: a group of 16 lanes reads 4 rows of 16 values, lane i
// giving the address of values 4 (i % 4) .. + 3 of row i / 4, and gets value i
// of the 4 rows.
__device__ __forceinline__ v4s lds_read_tr(const void* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p);
}

// 16 bytes a lane from base + off straight to LDS, lane after lane from `lds` on
// (both the same for the wavefront), and the wait for all of these loads.
__device__ __forceinline__ void lds_load16(const void* lds, const uint8_t* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)lds), "v"(off), "s"(base)
               : "m0", "memory");
}
__device__ __forceinline__ void lds_load_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ v8bf join_bf(v4s a, v4s b) {
  return __builtin_bit_cast(v8bf, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A wavefront's LDS writes before, its reads (of other lanes' data) after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ int64_t shfl64(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)__shfl((int)v, lane) | (uint64_t)(uint32_t)__shfl((int)(v >> 32), lane) << 32);
}

// The larger of two, NaN if either is (v_maximum3_f32): a NaN that a row sees
// stays in its maximum and its sum, so that its results are NaN however the tokens
// are split.  (v_max_f32 drops it and, where NaNs count, costs two instructions
// more to quiet its operands.)
__device__ __forceinline__ float attn_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A row that saw nothing has sum 0 and the running maximum's start, a finite
// number, so that no difference of maxima is a NaN.
constexpr float kNoMax = -__FLT_MAX__;

// The reference of a row's weights moves to a new maximum only when they would
// pass 2^kMaxStep: any reference serves that keeps them in range, and moving it
// costs a pass over the accumulators.
constexpr float kMaxStep = 8.0f;

// What scores, times scale, are taken less of before the exponential.
__device__ __forceinline__ float attn_shift(float top, float scale) { return top == kNoMax ? 0.0f : top * scale; }

// Page of token t of a sequence.  Nothing is made of it here, so that it can be
// on its way while a tile is worked on: kv_row() comes when the token's turn does.
__device__ __forceinline__ int token_page(const AttnArgs& a, int seq, int t) {
  const int32_t* table = t < a.prefix_len ? a.prefix_table : a.b.table + seq * a.b.ldt;
  return table[t >> a.c.page_shift];
}

// Bit j: a row at position p sees token t + j; live: bit shift + j, that token is there.
__device__ __forceinline__ unsigned long long row_sees(unsigned long long live, int p, int t, int shift, int window,
                                                       int sinks) {
  const int up = p - t, from = window > up ? 0 : up - window + 1, head = sinks - t;   // none of them wraps
  const unsigned long long before = up < 0 ? 0ull : up >= 63 ? ~0ull : (2ull << up) - 1;
  const unsigned long long after = from > 63 ? 0ull : ~0ull << from;
  const unsigned long long first = head <= 0 ? 0ull : head > 63 ? ~0ull : (1ull << head) - 1;
  return (live >> shift) & before & (after | first);
}

__device__ __forceinline__ float attn_lse(float m, float l, float scale) {
  return l != 0.0f ? (m * scale + __log2f(l)) * 0.69314718055994531f : -__builtin_inff();
}

}  // namespace sharq
