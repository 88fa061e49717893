// Paged key/value cache: appending rotated keys and values, and reading them
// back.  Both move every byte once and are bound by HBM bandwidth where rows are
// many: 7445 rows of 32 + 8 + 8 heads of 128 (bf16, 187 MB) 36 us, 5.2 TB/s; 20144
// into an MXFP4 cache 86 us (5.1 TB/s).  Read back: 22000 rows of 8 heads of 128 from
// a bf16 cache 38.5 us (4.7 TB/s); 20144 from an MXFP4 one 28.5 us, where a row's
// workgroup takes part of the cache lines that its neighbours take too, over
// several XCDs: 47 MB are fetched of 22 held.  An E4M3 cache: 8900 rows of 6 chunks
// of up to 2048, 32 + 8 + 8 heads of 128 (205 MB), 43 us, 4.8 TB/s; with the
// queries first, or a head a thread, 48.7; read back, 22000 rows as above, 38.7 us
// (3.5 TB/s).  One row takes 2.7 us, the chain of offsets, length, page table and
// store; the row's values are loaded beside it.
//
// Rotation of a head's pair (x_j, x_{j + D/2}) by the angle of its position:
//   y_j = x_j c_j - x_{j+D/2} s_j,  y_{j+D/2} = x_{j+D/2} c_j + x_j s_j,
// products and sums rounded to fp32 one by one.  The result is rounded once,
// to bf16 or (keys in an MXFP4 cache) straight to E2M1 under its block's
// scale: rounding it to bf16 first would only add an error.

#include "sharq_kv_device.hpp"

namespace sharq {

struct KvAppendArgs {
  const uint16_t *q, *k, *v;
  int64_t ldq, ldk, ldv;
  uint16_t* qo;
  int64_t ldqo;
  const float *cos, *sin;
  const int32_t* pos;
  int angles, q_heads, parts;   // rows of the angle tables; workgroups per row
  uint32_t rule_bias;
};

// Eight values -> one dword of codes under the scale of their block of 32 (this
// and the next three lanes of an aligned group of four); returns the scale code.
__device__ __forceinline__ uint32_t kv_quantize8(const float* x, uint32_t rule_bias, uint32_t& codes) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    m = a > m ? a : m;
  }
  uint32_t o = (uint32_t)__shfl_xor((int)m, 1);
  m = o > m ? o : m;
  o = (uint32_t)__shfl_xor((int)m, 2);
  m = o > m ? o : m;
  const int e = mx_exponent(m, rule_bias);
  codes = enc8(x, MxQ::make(e));
  return (uint32_t)(e + 127);
}

// A thread takes 8 values of a head's first half and the 8 that pair with them.
// Workgroup b: row b / parts, threads of its part of the row's heads.
template <int D, bool MX>
__global__ __launch_bounds__(kAppendThreads) void k_kv_append(KvAppendArgs a, KvBatchArgs b, KvCacheArgs c) {
  constexpr int kPer = D / 16;   // threads of a head
  const int row = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x % (unsigned)a.parts);
  const int item = part * kAppendThreads + (int)threadIdx.x;
  const int head = item / kPer, j = (item % kPer) * 8;
  const int kinds = a.q_heads + 2 * c.heads;
  // the row's values are on their way while its sequence is looked up
  const bool has = head < kinds;
  const bool is_q = head < a.q_heads, is_v = head >= a.q_heads + c.heads;
  const int h = is_q ? head : is_v ? head - a.q_heads - c.heads : head - a.q_heads;
  const uint16_t* src = is_q ? a.q + row * a.ldq : is_v ? a.v + row * a.ldv : a.k + row * a.ldk;
  uint4 x0{}, x1{};
  if (has) {
    x0 = *reinterpret_cast<const uint4*>(src + (int64_t)h * D + j);
    x1 = *reinterpret_cast<const uint4*>(src + (int64_t)h * D + j + D / 2);
  }
  const int s = find_seq(b, row);
  if (s >= b.seqs) return;   // behind the last sequence
  const SeqRows r = seq_rows(b, s);
  const int i = row - r.first, p = r.len - r.n + i;
  if (i < 0 || i >= r.n || p < 0) return;   // i is in range whenever the offsets do not decrease
  const int page = b.table[s * b.ldt + (p >> c.page_shift)];
  int angle = 0;
  if (a.cos) {
    angle = a.pos ? a.pos[row] : p;
    if (angle < 0 || angle >= a.angles) return;
  }
  float lo[8], hi[8];
  const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[2 * i] = bf16_lo(w0[i]), lo[2 * i + 1] = bf16_hi(w0[i]);
    hi[2 * i] = bf16_lo(w1[i]), hi[2 * i + 1] = bf16_hi(w1[i]);
  }
  if (a.cos && !is_v && has) {
    const float4* cp = reinterpret_cast<const float4*>(a.cos + (int64_t)angle * (D / 2) + j);
    const float4* sp = reinterpret_cast<const float4*>(a.sin + (int64_t)angle * (D / 2) + j);
    const float4 c0 = cp[0], c1 = cp[1], s0 = sp[0], s1 = sp[1];
    const float cs[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    const float sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = lo[i], w = hi[i];
      lo[i] = u * cs[i] - w * sn[i];
      hi[i] = w * cs[i] + u * sn[i];
    }
  }
  const int at = kv_row(page, p, c.pages, c.heads, is_q ? 0 : h, c.page_shift);
  if (MX && !is_q) {   // whole groups of four lanes reach this: a head has kPer of them, the same branch each
    uint32_t d0, d1;
    const uint32_t e0 = kv_quantize8(lo, a.rule_bias, d0), e1 = kv_quantize8(hi, a.rule_bias, d1);
    if (!has || at < 0) return;
    uint8_t* codes = (is_v ? c.v : c.k) + (int64_t)at * (D / 2);
    uint8_t* scale = (is_v ? c.vs : c.ks) + (int64_t)at * (D / 32);
    *reinterpret_cast<uint32_t*>(codes + j / 2) = d0;
    *reinterpret_cast<uint32_t*>(codes + j / 2 + D / 4) = d1;
    if (j % 32 == 0) {
      scale[j / 32] = (uint8_t)e0;
      scale[j / 32 + D / 64] = (uint8_t)e1;
    }
    return;
  }
  if (!has || (!is_q && at < 0)) return;
  uint16_t* dst = is_q ? a.qo + row * a.ldqo + (int64_t)h * D
                       : reinterpret_cast<uint16_t*>(is_v ? c.v : c.k) + (int64_t)at * D;
  *reinterpret_cast<uint4*>(dst + j) = make_uint4(bf16x2(lo[0], lo[1]), bf16x2(lo[2], lo[3]), bf16x2(lo[4], lo[5]),
                                                  bf16x2(lo[6], lo[7]));
  *reinterpret_cast<uint4*>(dst + j + D / 2) = make_uint4(bf16x2(hi[0], hi[1]), bf16x2(hi[2], hi[3]),
                                                          bf16x2(hi[4], hi[5]), bf16x2(hi[6], hi[7]));
}

// Values of dims j..j+N-1 and j+D/2..j+D/2+N-1 of a head, from bf16, N a multiple of 8.
template <int D, int N>
__device__ __forceinline__ void load_halves(const uint16_t* src, float* lo, float* hi) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    const uint4 x0 = *reinterpret_cast<const uint4*>(src + i), x1 = *reinterpret_cast<const uint4*>(src + i + D / 2);
    const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      lo[i + 2 * k] = bf16_lo(w0[k]), lo[i + 2 * k + 1] = bf16_hi(w0[k]);
      hi[i + 2 * k] = bf16_lo(w1[k]), hi[i + 2 * k + 1] = bf16_hi(w1[k]);
    }
  }
}

template <int N>
__device__ __forceinline__ void rotate_halves(const float* cp, const float* sp, float* lo, float* hi) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 c = *reinterpret_cast<const float4*>(cp + i), s = *reinterpret_cast<const float4*>(sp + i);
    const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float u = lo[i + k], w = hi[i + k];
      lo[i + k] = u * cs[k] - w * sn[k];
      hi[i + k] = w * cs[k] + u * sn[k];
    }
  }
}

// One wavefront: the keys or values of a head of one block of 16 tokens, of which tokens [from, from + n) are rows of
// the call from `row` on and, where `olds`, those before are in the cache.  Lane: token lane / 4, a quarter of both
// halves of the head.  The block's new scale is the larger of the one that its old tokens have and the one that the new
// ones need; where it grows, old codes are rounded again (exactly, but for those that become subnormal).
template <int D>
__device__ __forceinline__ void append8_block(const KvAppendArgs& a, const KvCacheArgs& c, bool is_v, int h, int at,
                                              int row, int pos, int from, int n, bool olds) {
  constexpr int N = D / 8;   // values of a half: 16 or 8
  const int lane = (int)threadIdx.x & 63, t = lane >> 2, j = (lane & 3) * N;
  uint8_t* const codes = (is_v ? c.v : c.k) + ((int64_t)at + t) * D + j;
  uint8_t* const scale = (is_v ? c.vs : c.ks) + at / kF8Block;
  bool mine = t >= from && t < from + n;
  const int r = row + (mine ? t - from : 0);
  float lo[N], hi[N];
  load_halves<D, N>((is_v ? a.v + r * a.ldv : a.k + r * a.ldk) + h * D + j, lo, hi);
  uint32_t old[2][N / 4] = {};
  bool was = olds && t < from;
  int before = kF8Least;
  if (olds) {   // on its way with the row's values, whether the scale grows or not
    const int held = (int)*scale - 127;
    if (was)
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        old[0][i] = reinterpret_cast<const uint32_t*>(codes)[i];
        old[1][i] = reinterpret_cast<const uint32_t*>(codes + D / 2)[i];
      }
    // no scale that an append leaves: the tokens before these were left out, and nothing of theirs is here
    if (held < kF8Least || held > kF8Most) was = false;
    else before = held;
  }
  if (a.cos) {
    const int angle = a.pos ? a.pos[r] : pos + (r - row);
    if (angle < 0 || angle >= a.angles) mine = false;   // left out
    if (!is_v && mine)
      rotate_halves<N>(a.cos + (int64_t)angle * (D / 2) + j, a.sin + (int64_t)angle * (D / 2) + j, lo, hi);
  }
  if (!__any(mine)) return;
  uint32_t peak = 0;   // of the finite values: one that is not does not take its neighbours with it
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t x = __float_as_uint(lo[i]) & 0x7FFFFFFFu, y = __float_as_uint(hi[i]) & 0x7FFFFFFFu;
    if (x < 0x7F800000u && x > peak) peak = x;
    if (y < 0x7F800000u && y > peak) peak = y;
  }
  if (!mine) peak = 0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)peak, d);
    peak = o > peak ? o : peak;
  }
  const int need = f8_exponent(peak, a.rule_bias), e = need > before ? need : before;
  if (was && e > before) {
    // a step of 20 takes the largest code to zero
    const float f = exp2_int(before - e < -30 ? -30 : before - e);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      reinterpret_cast<uint32_t*>(codes)[i] = f8_rescale4(old[0][i], f);
      reinterpret_cast<uint32_t*>(codes + D / 2)[i] = f8_rescale4(old[1][i], f);
    }
  }
  if (mine) {
    const float inv = exp2_int(-e);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      reinterpret_cast<uint32_t*>(codes)[i] = f8_encode4(lo + 4 * i, inv);
      reinterpret_cast<uint32_t*>(codes + D / 2)[i] = f8_encode4(hi + 4 * i, inv);
    }
  }
  if (lane == 0) *scale = (uint8_t)(e + 127);
}

// Appends to an E4M3 cache.  A scale is shared by 16 tokens of a page and head, so a block is one wavefront's, which
// the row that begins it finds: the first of a sequence's rows, or one at a multiple of 16.
template <int D>
__global__ __launch_bounds__(kAppend8Threads) void k_kv_append8(KvAppendArgs a, KvBatchArgs b, KvCacheArgs c,
                                                                unsigned first_query, int group) {
  const int tid = (int)threadIdx.x;
  if (blockIdx.x >= first_query) {
    // a thread: 8 values of a head's first half and the 8 that pair with them, of two heads: one lookup, one angle
    constexpr int kPer = D / 16;
    const int pair = kv_append8_pair(a.q_heads);
    const unsigned block = blockIdx.x - first_query;
    const unsigned item = block * kAppend8Threads + tid, per_row = (unsigned)pair * kPer;
    const int row = (int)(item / per_row), rest = (int)(item % per_row), h = rest / kPer, j = rest % kPer * 8;
    const int first = (int)((block * kAppend8Threads + (tid & ~63)) / per_row);   // of the wavefront
    if (first >= b.rows) return;
    float lo[2][8], hi[2][8];
    const bool has = row < b.rows, two = h + pair < a.q_heads;
    const int next = two ? pair * D : 0;
    if (has) {
      const uint16_t* const src = a.q + row * a.ldq + h * D + j;
      load_halves<D, 8>(src, lo[0], hi[0]);
      load_halves<D, 8>(src + next, lo[1], hi[1]);
    }
    int s = find_seq(b, first), past = b.seqs;   // few of a wavefront's threads are at a later row than the first
    if (!has) return;
    if (row == first) past = s;
    while (s < past) {
      const int mid = s + (past - s) / 2;
      if (b.offs[mid + 1] <= row) s = mid + 1;
      else past = mid;
    }
    if (s >= b.seqs) return;
    const SeqRows r = seq_rows(b, s);
    const int i = row - r.first, p = r.len - r.n + i;
    if (i < 0 || i >= r.n || p < 0) return;
    int angle = 0;
    if (a.cos) {
      angle = a.pos ? a.pos[row] : p;
      if (angle < 0 || angle >= a.angles) return;
    }
    const float *cp = a.cos + (int64_t)angle * (D / 2) + j, *sp = a.sin + (int64_t)angle * (D / 2) + j;
    uint16_t* const dst = a.qo + row * a.ldqo + h * D + j;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (a.cos) rotate_halves<8>(cp, sp, lo[k], hi[k]);
      if (k == 1 && !two) continue;
      uint16_t* const to = dst + k * next;
      *reinterpret_cast<uint4*>(to) = make_uint4(bf16x2(lo[k][0], lo[k][1]), bf16x2(lo[k][2], lo[k][3]),
                                                 bf16x2(lo[k][4], lo[k][5]), bf16x2(lo[k][6], lo[k][7]));
      *reinterpret_cast<uint4*>(to + D / 2) = make_uint4(bf16x2(hi[k][0], hi[k][1]), bf16x2(hi[k][2], hi[k][3]),
                                                         bf16x2(hi[k][4], hi[k][5]), bf16x2(hi[k][6], hi[k][7]));
    }
    return;
  }
  const unsigned block = blockIdx.x, parts = (unsigned)kv_append8_parts(c.heads);
  const int item = (int)(block % parts) * 4 + (tid >> 6), unit = (int)(block / parts);
  if (item >= 2 * c.heads) return;
  const bool is_v = item & 1;
  const int h = item >> 1;
  const int64_t end64 = ((int64_t)unit + 1) * group;
  const int end = end64 < b.rows ? (int)end64 : b.rows;
  int row = unit * group;
  while (row < end) {
    const int s = find_seq(b, row);
    if (s >= b.seqs) return;
    const SeqRows r = seq_rows(b, s);
    if (row < r.first || row >= r.first + r.n) return;   // offsets that decrease
    const int base = r.len - r.n, last = r.first + r.n;
    if (base + (row - r.first) < 0) row = -base < r.n ? r.first - base : last;   // rows at negative positions
    while (row < last && row < end) {
      const int p = base + (row - r.first), from = p & (kF8Block - 1);
      const int n = kF8Block - from < last - row ? kF8Block - from : last - row;
      if (row == r.first || from == 0) {
        const int page = b.table[s * b.ldt + (p >> c.page_shift)];
        const int at = kv_row(page, p & ~(kF8Block - 1), c.pages, c.heads, h, c.page_shift);
        if (at >= 0) append8_block<D>(a, c, is_v, h, at, row, p, from, n, from > 0);
      }
      row += n;
    }
  }
}

// A thread reads 8 values; workgroup b: row b / parts, as above.
template <int D, int F>
__global__ __launch_bounds__(kReadThreads) void k_kv_read(uint16_t* ko, int64_t ldk, uint16_t* vo, int64_t ldv,
                                                          int parts, KvBatchArgs b, KvCacheArgs c) {
  constexpr int kPer = D / 8;
  const int row = (int)(blockIdx.x / (unsigned)parts), part = (int)(blockIdx.x % (unsigned)parts);
  const int item = part * kReadThreads + (int)threadIdx.x;
  const int head = item / kPer, j = (item % kPer) * 8;
  const int s = find_seq(b, row);
  if (s >= b.seqs || head >= 2 * c.heads) return;
  const SeqRows r = seq_rows(b, s);
  const int i = row - r.first, p = r.len - r.n + i;
  if (i < 0 || i >= r.n) return;
  const bool is_v = head >= c.heads;
  const int h = is_v ? head - c.heads : head;
  const int at = p < 0 ? -1
                       : kv_row(b.table[s * b.ldt + (p >> c.page_shift)], p, c.pages, c.heads, h, c.page_shift);
  uint4 y{};
  if (at >= 0) {
    if (F == kKvMx) {
      const uint32_t codes = *reinterpret_cast<const uint32_t*>((is_v ? c.v : c.k) + (int64_t)at * (D / 2) + j / 2);
      y = mx_bf16x8(codes, (is_v ? c.vs : c.ks)[(int64_t)at * (D / 32) + j / 32]);
    } else if (F == kKvF8) {
      const uint2 codes = *reinterpret_cast<const uint2*>((is_v ? c.v : c.k) + (int64_t)at * D + j);
      y = f8_bf16x8(codes, (is_v ? c.vs : c.ks)[at / kF8Block]);
    } else {
      y = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(is_v ? c.v : c.k) + (int64_t)at * D + j);
    }
  }
  *reinterpret_cast<uint4*>((is_v ? vo + row * ldv : ko + row * ldk) + h * D + j) = y;
}

hipError_t launch_kv_append(const uint16_t* q, const uint16_t* k, const uint16_t* v, int64_t ldq, int64_t ldk,
                            int64_t ldv, int q_heads, uint16_t* qo, int64_t ldqo, const float* cos, const float* sin,
                            int angles, const int32_t* pos, uint32_t rule_bias, const KvBatchArgs& b,
                            const KvCacheArgs& c, int D, int fmt, int64_t max_rows, hipStream_t st) {
  const bool mx = fmt == kKvMx;
  KvAppendArgs a{q, k, v, ldq, ldk, ldv, qo, ldqo, cos, sin, pos, angles, q_heads, 0, rule_bias};
  if (fmt == kKvF8) {
    const int group = kv_append8_group(max_rows);
    const unsigned all = (unsigned)kv_append8_blocks(b.rows, max_rows, q_heads, c.heads, D);
    const unsigned first = all - (unsigned)kv_append8_queries(b.rows, q_heads, D);
    const dim3 g8(all), t8(kAppend8Threads);
    if (D == 128) k_kv_append8<128><<<g8, t8, 0, st>>>(a, b, c, first, group);
    else k_kv_append8<64><<<g8, t8, 0, st>>>(a, b, c, first, group);
    return hipGetLastError();
  }
  a.parts = kv_append_parts(q_heads, c.heads, D);
  const dim3 g((unsigned)b.rows * (unsigned)a.parts), t(kAppendThreads);
  if (D == 128)
    mx ? k_kv_append<128, true><<<g, t, 0, st>>>(a, b, c) : k_kv_append<128, false><<<g, t, 0, st>>>(a, b, c);
  else
    mx ? k_kv_append<64, true><<<g, t, 0, st>>>(a, b, c) : k_kv_append<64, false><<<g, t, 0, st>>>(a, b, c);
  return hipGetLastError();
}

template <int D>
static void kv_read(int fmt, dim3 g, uint16_t* ko, int64_t ldk, uint16_t* vo, int64_t ldv, int parts,
                    const KvBatchArgs& b, const KvCacheArgs& c, hipStream_t st) {
  const dim3 t(kReadThreads);
  if (fmt == kKvBf16) k_kv_read<D, kKvBf16><<<g, t, 0, st>>>(ko, ldk, vo, ldv, parts, b, c);
  else if (fmt == kKvMx) k_kv_read<D, kKvMx><<<g, t, 0, st>>>(ko, ldk, vo, ldv, parts, b, c);
  else k_kv_read<D, kKvF8><<<g, t, 0, st>>>(ko, ldk, vo, ldv, parts, b, c);
}

hipError_t launch_kv_read(uint16_t* ko, int64_t ldk, uint16_t* vo, int64_t ldv, const KvBatchArgs& b,
                          const KvCacheArgs& c, int D, int fmt, hipStream_t st) {
  const int parts = kv_read_parts(c.heads, D);
  const dim3 g((unsigned)b.rows * (unsigned)parts);
  if (D == 128) kv_read<128>(fmt, g, ko, ldk, vo, ldv, parts, b, c, st);
  else kv_read<64>(fmt, g, ko, ldk, vo, ldv, parts, b, c, st);
  return hipGetLastError();
}

}  // namespace sharq
