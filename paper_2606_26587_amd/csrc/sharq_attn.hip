// Attention over the paged cache: the kernels for many rows, and the launches of
// a call.

#include "sharq_attn_rows.hpp"

namespace sharq {

template <int D, bool MX, bool ALL>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_attn_rows(AttnArgs a, int tiles, int chunk_tiles, int first_slot) {
  __shared__ RowsLds<D> lds;
  attn_rows<D, MX, ALL>(a, (int)blockIdx.x, tiles, chunk_tiles, first_slot, lds);
}

template <int D, bool MX>
static void rows(bool all, dim3 g, const AttnArgs& a, int tiles, int chunk_tiles, int first_slot, hipStream_t st) {
  if (all) k_attn_rows<D, MX, true><<<g, 256, 0, st>>>(a, tiles, chunk_tiles, first_slot);
  else k_attn_rows<D, MX, false><<<g, 256, 0, st>>>(a, tiles, chunk_tiles, first_slot);
}

static hipError_t launch_attn_rows(const AttnArgs& a, int D, bool mx, bool all, const AttnSplit& s, int first_slot,
                                   hipStream_t st) {
  const dim3 g((unsigned)s.tiles * (unsigned)a.c.heads * (unsigned)s.chunks);
  if (D == 128)
    mx ? rows<128, true>(all, g, a, s.tiles, s.chunk_tiles, first_slot, st)
       : rows<128, false>(all, g, a, s.tiles, s.chunk_tiles, first_slot, st);
  else
    mx ? rows<64, true>(all, g, a, s.tiles, s.chunk_tiles, first_slot, st)
       : rows<64, false>(all, g, a, s.tiles, s.chunk_tiles, first_slot, st);
  return hipGetLastError();
}

hipError_t launch_attn_few(const AttnArgs& a, int D, bool mx, const AttnPlan& plan, hipStream_t st);
hipError_t launch_attn_shared(const AttnArgs& a, int D, bool mx, const AttnPlan& plan, hipStream_t st);
hipError_t launch_attn_merge(const AttnArgs& a, int D, hipStream_t st);

hipError_t launch_attention(const uint16_t* q, int64_t ldq, uint16_t* o, int64_t ldo, float* lse,
                            const KvBatchArgs& b, const KvCacheArgs& c, const AttnPlan& plan,
                            const int32_t* prefix_table, int prefix_len, int q_heads, int D, bool mx, int window,
                            int sinks, float scale, void* ws, hipStream_t st) {
  const int64_t items = (int64_t)b.rows * q_heads;
  AttnArgs a{q, ldq, o, ldo, lse, b, c, prefix_table, prefix_len, plan.shared ? prefix_len : 0, q_heads / c.heads,
             q_heads, window, sinks, (float)((double)scale * 1.4426950408889634),
             static_cast<float2*>(ws), nullptr, plan.slots};
  if (plan.slots) a.po = reinterpret_cast<float*>(static_cast<char*>(ws) + attn_ml_bytes(items, plan.slots));
  hipError_t e = hipSuccess;
  if (plan.shared && plan.few) {
    e = launch_attn_shared(a, D, mx, plan, st);
  } else {
    if (plan.shared) e = launch_attn_rows(a, D, mx, true, plan.prefix, plan.own.chunks, st);
    if (e != hipSuccess) return e;
    e = plan.few ? launch_attn_few(a, D, mx, plan, st) : launch_attn_rows(a, D, mx, false, plan.own, 0, st);
  }
  if (e != hipSuccess || plan.slots == 0) return e;
  return launch_attn_merge(a, D, st);
}

}  // namespace sharq
