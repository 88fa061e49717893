// Paged key/value cache: appending rotated keys and values, and reading them
// back.  Both move every byte once and are bound by HBM bandwidth where rows are
// many: 7445 rows of 32 + 8 + 8 heads of 128 (bf16, 187 MB) 36 us, 5.2 TB/s; 20144
// into an MXFP4 cache 86 us (5.1 TB/s).  Read back: 22000 rows of 8 heads of 128 from
// a bf16 cache 38.5 us (4.7 TB/s); 20144 from an MXFP4 one 28.5 us, where a row's
// workgroup takes part of the cache lines that its neighbours take too, over
// several XCDs: 47 MB are fetched of 22 held.  One row takes
// 2.7 us, the chain of offsets, length, page table and store; the row's values are
// loaded beside it.
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

// A thread reads 8 values; workgroup b: row b / parts, as above.
template <int D, bool MX>
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
    if (MX) {
      const uint32_t codes = *reinterpret_cast<const uint32_t*>((is_v ? c.v : c.k) + (int64_t)at * (D / 2) + j / 2);
      y = mx_bf16x8(codes, (is_v ? c.vs : c.ks)[(int64_t)at * (D / 32) + j / 32]);
    } else {
      y = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(is_v ? c.v : c.k) + (int64_t)at * D + j);
    }
  }
  *reinterpret_cast<uint4*>((is_v ? vo + row * ldv : ko + row * ldk) + h * D + j) = y;
}

hipError_t launch_kv_append(const uint16_t* q, const uint16_t* k, const uint16_t* v, int64_t ldq, int64_t ldk,
                            int64_t ldv, int q_heads, uint16_t* qo, int64_t ldqo, const float* cos, const float* sin,
                            int angles, const int32_t* pos, uint32_t rule_bias, const KvBatchArgs& b,
                            const KvCacheArgs& c, int D, bool mx, hipStream_t st) {
  KvAppendArgs a{q, k, v, ldq, ldk, ldv, qo, ldqo, cos, sin, pos, angles, q_heads, 0, rule_bias};
  a.parts = kv_append_parts(q_heads, c.heads, D);
  const dim3 g((unsigned)b.rows * (unsigned)a.parts), t(kAppendThreads);
  if (D == 128)
    mx ? k_kv_append<128, true><<<g, t, 0, st>>>(a, b, c) : k_kv_append<128, false><<<g, t, 0, st>>>(a, b, c);
  else
    mx ? k_kv_append<64, true><<<g, t, 0, st>>>(a, b, c) : k_kv_append<64, false><<<g, t, 0, st>>>(a, b, c);
  return hipGetLastError();
}

hipError_t launch_kv_read(uint16_t* ko, int64_t ldk, uint16_t* vo, int64_t ldv, const KvBatchArgs& b,
                          const KvCacheArgs& c, int D, bool mx, hipStream_t st) {
  const int parts = kv_read_parts(c.heads, D);
  const dim3 g((unsigned)b.rows * (unsigned)parts), t(kReadThreads);
  if (D == 128)
    mx ? k_kv_read<128, true><<<g, t, 0, st>>>(ko, ldk, vo, ldv, parts, b, c)
       : k_kv_read<128, false><<<g, t, 0, st>>>(ko, ldk, vo, ldv, parts, b, c);
  else
    mx ? k_kv_read<64, true><<<g, t, 0, st>>>(ko, ldk, vo, ldv, parts, b, c)
       : k_kv_read<64, false><<<g, t, 0, st>>>(ko, ldk, vo, ldv, parts, b, c);
  return hipGetLastError();
}

}  // namespace sharq
