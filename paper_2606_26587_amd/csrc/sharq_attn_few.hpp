// Attention over the paged cache where a sequence has few rows: single tokens
// and a few drafted ones.  What is read is nearly all keys and values, once, so
// the kernel is built to stream them from HBM.
//
// A workgroup takes the rows of one sequence that share a key/value head (its
// new tokens times the G query heads of that head, up to 16 NQ) and a range of
// its cached tokens; its four wavefronts take 32 NT tokens in turn and keep
// softmax states of their own, which are joined through LDS at the end.  Long
// sequences are split over several workgroups, whose partial results
// k_attn_merge joins.
//
// S^T = K Q^T and O^T = V^T P^T with 16x16x32 bf16 MFMAs: a lane holds four
// tokens of one row, so the rescaling needs no broadcast, and the accumulators
// of two 16-token products, rounded to bf16, are the P operand of one product
// over 32 tokens, if lane group g's eight k slots are taken as the tokens
// {4g..4g+3, 16+4g..16+4g+3}.  Keys go from HBM straight into their operand's
// registers (no byte is used by two lanes); values through a wavefront's
// own LDS for the transposing read.  An MXFP4 key's operand takes the k slots in
// the order that gives each lane D/4 consecutive values of its token: one load,
// one block scale.  An E4M3 key's takes 16 bytes of every 64; the 16 tokens of a
// group have one scale, which a lane reads beside the page of its token.
//
// A turn's loads are made without conditions on page bases in scalar registers,
// and the page table is read a turn ahead: with a wait for the table among the
// loads, 24 x 32768 tokens in MXFP4 took 180 us, now 128.  Measured with 8
// key/value heads of 128: 64 x up to 6000 tokens, window 4096, bf16: 178 us, 5.4
// TB/s (a 1 GiB copy: 5.16); 24 x up to 32768, MXFP4: 128 us, 4.6 TB/s, the
// dequantization and the products beside the stream; 32 x up to 16384, E4M3: 144
// us, 5.2 TB/s; one token over 8191: 9.6 us and 3.6 for the join (E4M3: 8 and 3),
// latencies of launch, table, keys and join.

#pragma once

#include "sharq_attn.hpp"

namespace sharq {

constexpr int kSub = 32;   // tokens of one pass through the two products

template <int D>
struct FewLds {
  uint4 v[4][kSub * D / 8];   // a wavefront's values; at the end the wavefronts' outputs
  float2 ml[4][16];
};

template <int D, int F, int NQ, int NT>
__device__ __forceinline__ void attn_few(const AttnArgs& a, int block, int chunk_tiles, int first_slot,
                                         FewLds<D>& shared) {
  constexpr bool MX = F == kKvMx, F8 = F == kKvF8;
  constexpr int kC = D / 8, kJ = D / 32, kDT = D / 16;
  constexpr int kTok = kSub * NT;            // tokens of a wavefront's turn
  constexpr int kG16 = 2 * NT;               // 16-token groups of a turn: each lies in one page
  auto& lds = shared.v;
  auto& lds_ml = shared.ml;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, col = lane & 15;
  const int head = block % a.c.heads;
  const int sc = block / a.c.heads, seq = sc % a.b.seqs, chunk = sc / a.b.seqs;
  const SeqRows sr = seq_rows(a.b, seq);
  if (sr.n == 0 || sr.n * a.group > 16 * NQ) return;
  const int base = sr.len - sr.n, rows = sr.n * a.group;
  const int p_hi = sr.len - 1;
  const KvSpan span = kv_span(a.t0, sr.len, base, p_hi, a.window, a.sinks, kTok);
  const int first = chunk * chunk_tiles, last = span.n < first + chunk_tiles ? span.n : first + chunk_tiles;

  // rows of this lane: row 16 n + col of the tile (the last one again past it)
  int grow[NQ], qh[NQ], p[NQ];
  v8bf qf[NQ][kJ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = 16 * n + col < rows ? 16 * n + col : rows - 1;
    grow[n] = sr.first + r / a.group, qh[n] = head * a.group + r % a.group, p[n] = base + r / a.group;
    const uint16_t* qp = a.q + (int64_t)grow[n] * a.ldq + (int64_t)qh[n] * D;
#pragma unroll
    for (int j = 0; j < kJ; ++j)
      qf[n][j] = *reinterpret_cast<const v8bf*>(qp + (MX   ? g * (D / 4) + 8 * j
                                                      : F8 ? 64 * (j >> 1) + 16 * g + 8 * (j & 1)
                                                           : 32 * j + 8 * g));
  }
  v4f o[NQ][kDT] = {};
  float m[NQ], l[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) m[n] = kNoMax, l[n] = 0.0f;

  // page of token (lane % kTok) of a turn, -1 where no row sees it (it may hold anything)
  auto page_of = [&](int ti) {
    const int t = kv_tile_start(span, a.t0, ti, kTok) + lane % kTok;
    return ti < last && t < span.hi && (t >= span.low || t < a.sinks) ? token_page(a, seq, t) : -1;
  };
  uint4* const v_lds = lds[wave];
  const int v_tok = mx_token<D>(lane);   // MXFP4: the token of 16 whose values this lane brings
  int v_at[kDT];   // this lane's reads of the values' tile; 16 tokens further on is a constant away
#pragma unroll
  for (int d = 0; d < kDT; ++d)
    v_at[d] = 16 * kv_chunk<D>(4 * g + (col >> 2), 2 * d + ((lane & 3) >> 1)) + 8 * (lane & 1);
  int next = page_of(first + wave);
  for (int ti = first + wave; ti < last; ti += 4) {
    const int ts = kv_tile_start(span, a.t0, ti, kTok);
    const int at = kv_row(next, ts + lane % kTok, a.c.pages, a.c.heads, head, a.c.page_shift);
    const unsigned long long live = __ballot(at >= 0);
    // whether every row sees every token of the turn
    const bool whole = live == ~0ull && ts + kTok - 1 <= base &&
                       (p_hi - ts < a.window || ts + kTok <= a.sinks);
    next = page_of(ti + 4);
    if (live == 0) continue;
    // Every load is made: a token that no row sees takes its place in its page, and a group without a page takes
    // another's.  Keys there are masked, values set to zero.
    constexpr int kKeys = MX ? 1 : F8 ? D / 64 : kJ, kVals = MX ? 1 : F8 ? D / 64 : kC / 4;
    uint4 kb[kG16][kKeys], vb[kG16][kVals];
    uint32_t ke[kG16], ve[kG16];
    const int l1 = __builtin_ctzll(live), any = __builtin_amdgcn_readlane(at, l1) - (l1 & 15);
    uint32_t kse = 0, vse = 0;   // E4M3: lane i holds the scales of token i's block
    if (F8) {
      const uint32_t block = (uint32_t)(at >= 0 ? at : any) / kF8Block;
      kse = a.c.ks[block], vse = a.c.vs[block];
    }
#pragma unroll
    for (int i = 0; i < kG16; ++i) {
      const unsigned mine = (unsigned)(live >> (16 * i)) & 0xFFFFu;
      const int l0 = 16 * i + (mine ? __builtin_ctz(mine) : 0);
      const int64_t row = mine ? __builtin_amdgcn_readlane(at, l0) - (l0 & 15) : any;
      if (MX) {
        const uint8_t *kp = a.c.k + row * (D / 2), *vp = a.c.v + row * (D / 2);
        const uint8_t *ksp = a.c.ks + row * (D / 32), *vsp = a.c.vs + row * (D / 32);
        // a quarter g of a token: the operand's for the keys, for the values one that suits the LDS
        const uint32_t ko = (uint32_t)(col * (D / 2) + g * (D / 8)), vo = (uint32_t)(v_tok * (D / 2) + g * (D / 8));
        if (D == 128) {
          kb[i][0] = *reinterpret_cast<const uint4*>(kp + ko);
          vb[i][0] = *reinterpret_cast<const uint4*>(vp + vo);
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(kp + ko), y = *reinterpret_cast<const uint2*>(vp + vo);
          kb[i][0] = make_uint4(x.x, x.y, 0, 0), vb[i][0] = make_uint4(y.x, y.y, 0, 0);
        }
        ke[i] = ksp[(uint32_t)(col * (D / 32) + g * (D / 32) / 4)];
        ve[i] = vsp[(uint32_t)(v_tok * (D / 32) + g * (D / 32) / 4)];
      } else if (F8) {
        const uint8_t *kp = a.c.k + row * D, *vp = a.c.v + row * D;
#pragma unroll
        for (int j = 0; j < kKeys; ++j) {
          kb[i][j] = *reinterpret_cast<const uint4*>(kp + (uint32_t)(col * D + 16 * g) + 64 * j);
          vb[i][j] = *reinterpret_cast<const uint4*>(vp + (uint32_t)(f8_token(lane) * D + 16 * (lane & 3)) + 64 * j);
        }
        ke[i] = (uint32_t)__builtin_amdgcn_readlane((int)kse, l0);
        ve[i] = (uint32_t)__builtin_amdgcn_readlane((int)vse, l0);
      } else {
        const uint8_t *kp = a.c.k + row * (D * 2), *vp = a.c.v + row * (D * 2);
#pragma unroll
        for (int j = 0; j < kJ; ++j) kb[i][j] = *reinterpret_cast<const uint4*>(kp + (uint32_t)(col * D * 2 + 16 * g) + 64 * j);
#pragma unroll
        for (int j = 0; j < kC / 4; ++j) vb[i][j] = *reinterpret_cast<const uint4*>(vp + (uint32_t)(lane * 16) + 1024 * j);
      }
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      v4f s[NQ][2] = {};
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          uint4 kx;
          if (MX) {
            const uint4& w = kb[2 * u + mt][0];
            kx = mx_bf16x8(j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w, ke[2 * u + mt]);
          } else if (F8) {
            const uint4& w = kb[2 * u + mt][j >> 1];
            kx = f8_bf16x8(j & 1 ? make_uint2(w.z, w.w) : make_uint2(w.x, w.y), ke[2 * u + mt]);
          } else {
            kx = kb[2 * u + mt][j];
          }
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            s[n][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, kx), qf[n][j], s[n][mt], 0, 0, 0);
        }
      wave_sync();   // the reads of the turn before are done
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        const int i = 2 * u + mt;
        const unsigned mine = (unsigned)(live >> (16 * i)) & 0xFFFFu;
        if (MX) {
          const int t = v_tok, c0 = g * (D / 32);
          const uint32_t w[4] = {vb[i][0].x, vb[i][0].y, vb[i][0].z, vb[i][0].w};
          const bool dead = !((mine >> t) & 1);
#pragma unroll
          for (int e = 0; e < D / 32; ++e)   // zero codes times 2^-127
            v_lds[16 * mt * kC + kv_chunk<D>(t, c0 + e)] = mx_bf16x8(dead ? 0 : w[e], dead ? 0 : ve[i]);
        } else if (F8) {
#pragma unroll
          for (int j = 0; j < kVals; ++j) {
            const int t = f8_token(lane), c0 = 8 * j + 2 * (lane & 3);
            const bool dead = !((mine >> t) & 1);
            const uint4 x = vb[i][j];
            const uint32_t e = dead ? 127 : ve[i];
            v_lds[16 * mt * kC + kv_chunk<D>(t, c0)] = f8_bf16x8(dead ? make_uint2(0, 0) : make_uint2(x.x, x.y), e);
            v_lds[16 * mt * kC + kv_chunk<D>(t, c0 + 1)] = f8_bf16x8(dead ? make_uint2(0, 0) : make_uint2(x.z, x.w), e);
          }
        } else {
#pragma unroll
          for (int j = 0; j < kC / 4; ++j) {
            const int t = j * (64 / kC) + lane / kC;
            uint4 x = vb[i][j];
            if (!((mine >> t) & 1)) x = make_uint4(0, 0, 0, 0);
            v_lds[16 * mt * kC + kv_chunk<D>(t, lane % kC)] = x;
          }
        }
      }
      wave_sync();
      v8bf pf[NQ];
      float top[NQ];
      bool moved = false;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        if (!whole) {
          const uint32_t see = (uint32_t)(row_sees(live, p[n], ts + 4 * g, 4 * g, a.window, a.sinks) >> (kSub * u));
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[n][mt][i] = see & (1u << (16 * mt + i)) ? s[n][mt][i] : -__builtin_inff();
        }
        top[n] = attn_max(attn_max(attn_max(s[n][0][0], s[n][0][1]), attn_max(s[n][0][2], s[n][0][3])),
                       attn_max(attn_max(s[n][1][0], s[n][1][1]), attn_max(s[n][1][2], s[n][1][3])));
        top[n] = attn_max(top[n], __shfl_xor(top[n], 16));
        top[n] = attn_max(top[n], __shfl_xor(top[n], 32));
        moved |= (top[n] - m[n]) * a.scale > kMaxStep;
      }
      if (__any(moved)) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          top[n] = attn_max(top[n], m[n]);
          const float alpha = __builtin_amdgcn_exp2f((m[n] - top[n]) * a.scale);
          m[n] = top[n];
          l[n] *= alpha;
#pragma unroll
          for (int d = 0; d < kDT; ++d) o[n][d] *= alpha;
        }
      }
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float shift = attn_shift(m[n], a.scale);
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i >> 2][i & 3], a.scale, -shift));
          l[n] += e[i];
        }
        pf[n] = __builtin_bit_cast(v8bf, make_uint4(bf16x2(e[0], e[1]), bf16x2(e[2], e[3]), bf16x2(e[4], e[5]),
                                                    bf16x2(e[6], e[7])));
      }
#pragma unroll
      for (int d = 0; d < kDT; ++d) {
        const char* from = reinterpret_cast<const char*>(v_lds) + v_at[d];
        const v8bf vf = join_bf(lds_read_tr(from), lds_read_tr(from + 16 * kC * 16));
#pragma unroll
        for (int n = 0; n < NQ; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], o[n][d], 0, 0, 0);
      }
    }
  }

  // the four wavefronts' states joined, 16 rows at a time; D fp32 values of a row take D / 4 chunks of 16 bytes
  float4* const o_lds = reinterpret_cast<float4*>(lds[0]);   // [4][16][D / 4], as large as the values' tiles
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l[n] += __shfl_xor(l[n], 16);
    l[n] += __shfl_xor(l[n], 32);
    __syncthreads();
    if (g == 0) lds_ml[wave][col] = make_float2(m[n], l[n]);
#pragma unroll
    for (int d = 0; d < kDT; ++d)   // exchanged by row, so that 16 rows at one chunk use all banks
      o_lds[(wave * 16 + col) * (D / 4) + ((4 * d + g) ^ col)] = make_float4(o[n][d][0], o[n][d][1], o[n][d][2], o[n][d][3]);
    __syncthreads();
    for (int i = tid; i < 16 * (D / 4); i += 256) {
      const int r = i / (D / 4), ch = i % (D / 4), row = 16 * n + r;
      if (row >= rows) continue;
      float2 s[4];
      float top = kNoMax;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        s[w] = lds_ml[w][r];
        top = attn_max(top, s[w].x);
      }
      float sum = 0.0f, x0 = 0.0f, x1 = 0.0f, x2 = 0.0f, x3 = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f((s[w].x - top) * a.scale);
        const float4 x = o_lds[(w * 16 + r) * (D / 4) + (ch ^ r)];
        sum += f * s[w].y, x0 += f * x.x, x1 += f * x.y, x2 += f * x.z, x3 += f * x.w;
      }
      const int64_t row_g = sr.first + row / a.group;
      const int h = head * a.group + row % a.group;
      if (a.slots) {
        const int64_t at = ((int64_t)(first_slot + chunk) * a.b.rows + row_g) * a.q_heads + h;
        if (ch == 0) a.ml[at] = make_float2(top, sum);
        if (sum != 0.0f) *reinterpret_cast<float4*>(a.po + at * D + 4 * ch) = make_float4(x0, x1, x2, x3);
      } else {
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        *reinterpret_cast<uint2*>(a.o + row_g * a.ldo + (int64_t)h * D + 4 * ch) =
            make_uint2(bf16x2(x0 * inv, x1 * inv), bf16x2(x2 * inv, x3 * inv));
        if (a.lse && ch == 0) a.lse[row_g * a.q_heads + h] = attn_lse(top, sum, a.scale);
      }
    }
  }
}

}  // namespace sharq
