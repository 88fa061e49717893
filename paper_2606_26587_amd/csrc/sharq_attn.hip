// Attention over the paged cache: the kernels for many rows, and the launches of
// a call.

#include "sharq_attn_rows.hpp"

namespace sharq {

constexpr int kCus = 256;

template <int D, bool MX>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_attn_rows(AttnArgs a, int tiles, int chunk_tiles) {
  __shared__ RowsLds<D> lds;
  // Late tiles of a sequence see most tokens and come first.  Where all workgroups run at once, two on a CU, the second
  // 256 come in the other order, so that the longest share their CUs with the shortest: 2 x
  // 1024 tokens, 32 and 8 heads of 128, 30.0 and 28.5 us, 2048 behind 6144 250 and 245, 4 x 500 22.6 and 23.1.
  int block = (int)blockIdx.x;
  const int heads = a.c.heads, half = kCus / heads;
  if ((int)gridDim.x == tiles * heads && tiles * heads <= 2 * kCus && block >= half * heads)
    block = (tiles - 1 - (block / heads - half)) * heads + block % heads;
  attn_rows<D, MX, false>(a, block, tiles, chunk_tiles, 0, lds);
}

static hipError_t launch_attn_rows(const AttnArgs& a, int D, bool mx, const AttnSplit& s, hipStream_t st) {
  const dim3 g((unsigned)s.tiles * (unsigned)a.c.heads * (unsigned)s.chunks);
  if (D == 128)
    mx ? k_attn_rows<128, true><<<g, 256, 0, st>>>(a, s.tiles, s.chunk_tiles)
       : k_attn_rows<128, false><<<g, 256, 0, st>>>(a, s.tiles, s.chunk_tiles);
  else
    mx ? k_attn_rows<64, true><<<g, 256, 0, st>>>(a, s.tiles, s.chunk_tiles)
       : k_attn_rows<64, false><<<g, 256, 0, st>>>(a, s.tiles, s.chunk_tiles);
  return hipGetLastError();
}

hipError_t launch_attn_few(const AttnArgs& a, int D, bool mx, const AttnPlan& plan, hipStream_t st);
hipError_t launch_attn_mixed(const AttnArgs& a, int D, const AttnPlan& plan, hipStream_t st);
hipError_t launch_attn_shared(const AttnArgs& a, int D, bool mx, const AttnPlan& plan, hipStream_t st);
hipError_t launch_attn_merge(const AttnArgs& a, int D, hipStream_t st);

hipError_t launch_attention(const uint16_t* q, int64_t ldq, uint16_t* o, int64_t ldo, float* lse,
                            const KvBatchArgs& b, const KvCacheArgs& c, const AttnPlan& plan,
                            const int32_t* prefix_table, int prefix_len, int q_heads, int D, bool mx, int window,
                            int sinks, float scale, void* ws, hipStream_t st) {
  const int64_t items = (int64_t)b.rows * q_heads;
  AttnArgs a{q, ldq, o, ldo, lse, b, c, prefix_table, prefix_len, plan.shared ? prefix_len : 0,
             plan.mixed ? 16 : 0, q_heads / c.heads, q_heads, window, sinks,
             (float)((double)scale * 1.4426950408889634), static_cast<float2*>(ws), nullptr, plan.slots};
  if (plan.slots) a.po = reinterpret_cast<float*>(static_cast<char*>(ws) + attn_ml_bytes(items, plan.slots));
  const hipError_t e = plan.shared  ? launch_attn_shared(a, D, mx, plan, st)
                       : plan.mixed ? launch_attn_mixed(a, D, plan, st)
                       : plan.few   ? launch_attn_few(a, D, mx, plan, st)
                                    : launch_attn_rows(a, D, mx, plan.own, st);
  if (e != hipSuccess || plan.slots == 0) return e;
  return launch_attn_merge(a, D, st);
}

}  // namespace sharq
