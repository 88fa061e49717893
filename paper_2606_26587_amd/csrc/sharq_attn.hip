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
  int group, q_heads, window, sinks, tiles;
  float scale;   // of the scores, times log2 e
};

constexpr int kT = 64;        // tokens of a key/value tile
constexpr int kRowsA = 128;   // rows of a workgroup: 32 a wavefront

// Position of 16-byte chunk c of token t's row in an LDS tile.  The keys are
// read 16 tokens at a time at one chunk, the values 4 tokens at a time at 64
// consecutive bytes: under this exchange of chunks both fall on all 64 banks.
template <int D>
__device__ __forceinline__ int kv_chunk(int t, int c) {
  constexpr int kC = D / 8;
  const int f = D == 128 ? ((t & 3) << 2 | ((t >> 2) & 3)) : (((t >> 1) & 1) << 2 | ((t >> 2) & 3));
  return t * kC + (c ^ f);
}

// Sequence and tile of work unit `unit` of tiles of kRowsA rows; false: none.
__device__ __forceinline__ bool find_tile(const KvBatchArgs& b, int group, int unit, int& seq, int& tile) {
  const int lane = (int)(threadIdx.x & 63);
  int base = 0;
  for (int s0 = 0; s0 < b.seqs; s0 += 64) {
    const int s = s0 + lane;
    int n = 0;
    if (s < b.seqs) n = (int)(((int64_t)seq_rows(b, s).n * group + kRowsA - 1) / kRowsA);
    int sum = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    const unsigned long long past = __ballot(base + sum > unit);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      seq = s0 + l;
      tile = unit - base - (__shfl(sum, l) - __shfl(n, l));
      return true;
    }
    base += __shfl(sum, 63);
  }
  return false;
}

template <int D, bool MX>
__global__ __launch_bounds__(256, 2) void k_attn(AttnArgs a) {
  constexpr int kC = D / 8, kDT = D / 32;   // 16-byte chunks of a row, 32-wide tiles of D
  __shared__ uint4 sk[kT * kC], sv[kT * kC];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  // heads fastest: workgroups are dealt to the XCDs in turn, so each L2 sees few heads' keys and values.
  // Late tiles of a sequence, which see most tokens, first.
  const int head = (int)(blockIdx.x % (unsigned)a.c.heads);
  const int unit = a.tiles - 1 - (int)(blockIdx.x / (unsigned)a.c.heads);
  int seq, tile;
  if (!find_tile(a.b, a.group, unit, seq, tile)) return;
  const SeqRows sr = seq_rows(a.b, seq);
  const int base = sr.len - sr.n;                       // position of the sequence's first row
  const int rows = (int)((int64_t)sr.n * a.group - (int64_t)tile * kRowsA < kRowsA
                             ? (int64_t)sr.n * a.group - (int64_t)tile * kRowsA : kRowsA);
  // this lane's row (the last one again where the tile is not full)
  const int rr = wave * 32 + (lane & 31);
  const int64_t r = (int64_t)tile * kRowsA + (rr < rows ? rr : rows - 1);
  const int token = (int)(r / a.group), qh = head * a.group + (int)(r % a.group);
  const int p = base + token;
  const int p_lo = base + (int)((int64_t)tile * kRowsA / a.group);
  const int p_hi = base + (int)(((int64_t)tile * kRowsA + rows - 1) / a.group);

  v8bf qf[D / 16];
  {
    const uint16_t* qp = a.q + (int64_t)(sr.first + token) * a.ldq + (int64_t)qh * D + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) qf[i] = *reinterpret_cast<const v8bf*>(qp + 16 * i);
  }
  v16f o[kDT] = {};
  float m = -__FLT_MAX__, l = 0.0f;

  for (int part = 0; part < 2; ++part) {
    const int t0 = part ? a.prefix_len : 0, t1 = part ? sr.len : (a.prefix_len < sr.len ? a.prefix_len : sr.len);
    const int32_t* table = part ? a.b.table + seq * a.b.ldt : a.prefix_table;
    const KvSpan span = kv_span(t0, t1, p_lo, p_hi, a.window, a.sinks, kT);
    for (int ti = 0; ti < span.n; ++ti) {
      const int ts = kv_tile_start(span, t0, ti, kT);
      // lane i: cache row of token ts + i, -1 where no row of the tile sees it (it may hold anything)
      const int t = ts + lane;
      int at = -1;
      if (t < span.hi && (t >= span.low || t < a.sinks))
        at = kv_row(table[t >> a.c.page_shift], t, a.c.pages, a.c.heads, head, a.c.page_shift);
      const unsigned long long live = __ballot(at >= 0);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kT * kC / 256; ++i) {
        const int id = i * 256 + tid, row = id / kC, ch = id % kC;
        const int64_t src = __shfl(at, row);
        uint4 kx{}, vx{};
        if (src >= 0) {
          if (MX) {
            kx = mx_bf16x8(*reinterpret_cast<const uint32_t*>(a.c.k + src * (D / 2) + ch * 4),
                           a.c.ks[src * (D / 32) + ch / 4]);
            vx = mx_bf16x8(*reinterpret_cast<const uint32_t*>(a.c.v + src * (D / 2) + ch * 4),
                           a.c.vs[src * (D / 32) + ch / 4]);
          } else {
            kx = *reinterpret_cast<const uint4*>(a.c.k + src * (D * 2) + ch * 16);
            vx = *reinterpret_cast<const uint4*>(a.c.v + src * (D * 2) + ch * 16);
          }
        }
        sk[kv_chunk<D>(row, ch)] = kx;
        sv[kv_chunk<D>(row, ch)] = vx;
      }
      __syncthreads();
      v16f s[2] = {};
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const v8bf kf = *reinterpret_cast<const v8bf*>(&sk[kv_chunk<D>(mt * 32 + (lane & 31), 2 * i + half)]);
          s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i], s[mt], 0, 0, 0);
        }
      float top = m;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = mt * 32 + 8 * (i >> 2) + 4 * half + (i & 3), tt = ts + j;
          const bool seen = ((live >> j) & 1) && tt <= p && (p - tt < a.window || tt < a.sinks);
          s[mt][i] = seen ? s[mt][i] : -__builtin_inff();
          top = fmaxf(top, s[mt][i]);
        }
      top = fmaxf(top, __shfl_xor(top, 32));
      const float shift = top * a.scale, alpha = __builtin_amdgcn_exp2f(m * a.scale - shift);
      m = top;
      float sum = 0.0f;
      v8bf pf[4];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][i], a.scale, -shift));
          sum += e;
          pf[2 * mt + (i >> 3)][i & 7] = (__bf16)e;
        }
      l = l * alpha + sum;
#pragma unroll
      for (int d = 0; d < kDT; ++d) o[d] *= alpha;
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
          v4s x[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            // a group of 16 lanes reads 4 tokens x 16 values; lane i gets value i of the 4 tokens
            const int tok = 16 * st + 8 * u + 4 * half + ((lane & 15) >> 2);
            const int ch = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            const char* at_lds = reinterpret_cast<const char*>(&sv[kv_chunk<D>(tok, ch)]) + 8 * (lane & 1);
            x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at_lds));
          }
          const v8bf vf = __builtin_bit_cast(v8bf, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[st], o[d], 0, 0, 0);
        }
    }
  }
  l += __shfl_xor(l, 32);
  if (rr >= rows) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  uint16_t* op = a.o + (int64_t)(sr.first + token) * a.ldo + (int64_t)qh * D;
#pragma unroll
  for (int d = 0; d < kDT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(op + 32 * d + 8 * i + 4 * half) =
          make_uint2(bf16x2(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), bf16x2(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
  if (a.lse && half == 0)
    a.lse[(int64_t)(sr.first + token) * a.q_heads + qh] =
        l > 0.0f ? (m * a.scale + __log2f(l)) * 0.69314718055994531f : -__builtin_inff();
}

hipError_t launch_attention(const uint16_t* q, int64_t ldq, uint16_t* o, int64_t ldo, float* lse,
                            const KvBatchArgs& b, const KvCacheArgs& c, int max_rows, const int32_t* prefix_table,
                            int prefix_len, int q_heads, int D, bool mx, int window, int sinks, float scale,
                            hipStream_t st) {
  const int group = q_heads / c.heads;
  // no sequence has more than max_rows rows, and all together have no more than b.rows
  const int64_t most = (int64_t)b.seqs * (((int64_t)max_rows * group + kRowsA - 1) / kRowsA);
  const int64_t packed = (int64_t)b.rows * group / kRowsA + b.seqs;
  const AttnArgs a{q, ldq, o, ldo, lse, b, c, prefix_table, prefix_len, group, q_heads, window, sinks,
                   (int)(most < packed ? most : packed), (float)((double)scale * 1.4426950408889634)};
  const dim3 g((unsigned)a.tiles * (unsigned)c.heads), t(256);
  if (D == 128)
    mx ? k_attn<128, true><<<g, t, 0, st>>>(a) : k_attn<128, false><<<g, t, 0, st>>>(a);
  else
    mx ? k_attn<64, true><<<g, t, 0, st>>>(a) : k_attn<64, false><<<g, t, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace sharq
