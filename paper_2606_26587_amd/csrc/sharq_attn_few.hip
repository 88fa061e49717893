// Attention over the paged cache: the kernels for few rows, and the kernel that
// joins partial results.

#include "sharq_attn_few.hpp"

namespace sharq {

template <int D, bool MX, int NQ, int NT>
__global__ __launch_bounds__(256, 2) void k_attn_few(AttnArgs a, int chunk_tiles, int first_slot) {
  __shared__ FewLds<D> lds;
  attn_few<D, MX, NQ, NT>(a, (int)blockIdx.x, chunk_tiles, first_slot, lds);
}

// Joins the partial results of a row and head.  D / 4 threads form a group; WIDE
// false: a group for each item takes all of its few slots; true: all groups of a
// workgroup share one item's many slots.  Eight slots' states and outputs are on
// their way together (what a slot that saw nothing left unwritten is read and
// dropped).  Sums are formed in a fixed order: the same call gives the same bits.
// 32 items of 64 slots: 3.6 us (7.0 with a slot's output read only once its state
// had come); 2048 items of 17 slots: 6.2 us, 8.8 MB of states and outputs.
template <int D, bool WIDE>
__global__ __launch_bounds__(256) void k_attn_merge(AttnArgs a) {
  constexpr int kPer = D / 4, kG = 256 / kPer, kTrip = 8;
  __shared__ float4 lds_o[WIDE ? kG : 1][WIDE ? kPer : 1];
  __shared__ float2 lds_s[WIDE ? kG : 1];
  const int64_t all = (int64_t)a.b.rows * a.q_heads;
  const int grp = (int)threadIdx.x / kPer, ch = (int)threadIdx.x % kPer;
  const int64_t items = (int64_t)kv_clamp(a.b.offs[a.b.seqs], 0, a.b.rows) * a.q_heads;   // without padding rows
  for (int64_t i0 = blockIdx.x; i0 * (WIDE ? 1 : kG) < items; i0 += gridDim.x) {
    const int64_t item = WIDE ? i0 : i0 * kG + grp;
    float top = kNoMax, sum = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (WIDE || item < items)
      for (int s0 = WIDE ? grp : 0; s0 < a.slots; s0 += kTrip * (WIDE ? kG : 1)) {
        float2 t[kTrip];
        float4 x[kTrip];
#pragma unroll
        for (int i = 0; i < kTrip; ++i) {
          const int s = s0 + i * (WIDE ? kG : 1);
          t[i] = make_float2(kNoMax, 0.0f);
          if (s < a.slots) {
            const int64_t at = s * all + item;
            t[i] = a.ml[at];
            x[i] = *reinterpret_cast<const float4*>(a.po + at * D + 4 * ch);
          }
        }
        float now = top;
#pragma unroll
        for (int i = 0; i < kTrip; ++i) now = t[i].y != 0.0f ? attn_max(now, t[i].x) : now;
        const float f = __builtin_amdgcn_exp2f((top - now) * a.scale);
        sum *= f, o.x *= f, o.y *= f, o.z *= f, o.w *= f;
        top = now;
#pragma unroll
        for (int i = 0; i < kTrip; ++i) {
          if (t[i].y == 0.0f) continue;   // it saw nothing (a sum that is NaN did)
          const float e = __builtin_amdgcn_exp2f((t[i].x - now) * a.scale);
          sum += e * t[i].y;
          o.x += e * x[i].x, o.y += e * x[i].y, o.z += e * x[i].z, o.w += e * x[i].w;
        }
      }
    if (WIDE) {
      __syncthreads();   // the item before is done with
      lds_o[grp][ch] = o;
      if (ch == 0) lds_s[grp] = make_float2(top, sum);
      __syncthreads();
      if (grp != 0) continue;
      top = kNoMax, sum = 0.0f, o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < kG; ++i) top = attn_max(top, lds_s[i].x);
#pragma unroll
      for (int i = 0; i < kG; ++i) {
        const float e = __builtin_amdgcn_exp2f((lds_s[i].x - top) * a.scale);
        const float4 x = lds_o[i][ch];
        sum += e * lds_s[i].y;
        o.x += e * x.x, o.y += e * x.y, o.z += e * x.z, o.w += e * x.w;
      }
    } else if (item >= items) {
      continue;
    }
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    const int64_t row = item / a.q_heads, h = item % a.q_heads;
    *reinterpret_cast<uint2*>(a.o + row * a.ldo + h * D + 4 * ch) =
        make_uint2(bf16x2(o.x * inv, o.y * inv), bf16x2(o.z * inv, o.w * inv));
    if (a.lse && ch == 0) a.lse[item] = attn_lse(top, sum, a.scale);
  }
}

template <int D, bool MX>
static void few(int nq, dim3 g, const AttnArgs& a, int chunk_tiles, hipStream_t st) {
  constexpr int NT = MX ? 2 : 1;
  if (nq == 1) k_attn_few<D, MX, 1, NT><<<g, 256, 0, st>>>(a, chunk_tiles, 0);
  if constexpr (D == 64 || MX)
    if (nq == 2) k_attn_few<D, MX, 2, NT><<<g, 256, 0, st>>>(a, chunk_tiles, 0);
  if constexpr (D == 64 && MX)
    if (nq == 4) k_attn_few<D, MX, 4, NT><<<g, 256, 0, st>>>(a, chunk_tiles, 0);
}

hipError_t launch_attn_few(const AttnArgs& a, int D, bool mx, const AttnPlan& plan, hipStream_t st) {
  const dim3 g((unsigned)plan.own.chunks * (unsigned)a.b.seqs * (unsigned)a.c.heads);
  const int nq = plan.few, ct = plan.own.chunk_tiles;
  if (D == 128) mx ? few<128, true>(nq, g, a, ct, st) : few<128, false>(nq, g, a, ct, st);
  else mx ? few<64, true>(nq, g, a, ct, st) : few<64, false>(nq, g, a, ct, st);
  return hipGetLastError();
}

// Many items fill the chip with a group each: with 8 or 9 slots, 12000 items took
// 31 us wide and 6 us otherwise; 32 items of 64 slots are the other end.
constexpr int64_t kWideItems = 1024;

template <int D>
static void merge(const AttnArgs& a, hipStream_t st) {
  const int64_t items = (int64_t)a.b.rows * a.q_heads, most = 1 << 20;
  const bool wide = a.slots > 8 && items <= kWideItems;
  const int64_t g = wide ? items : ceil_div(items, 256 / (D / 4));
  const unsigned grid = (unsigned)(g < most ? g : most);
  if (wide) k_attn_merge<D, true><<<grid, 256, 0, st>>>(a);
  else k_attn_merge<D, false><<<grid, 256, 0, st>>>(a);
}

hipError_t launch_attn_merge(const AttnArgs& a, int D, hipStream_t st) {
  if (D == 128) merge<128>(a, st);
  else merge<64>(a, st);
  return hipGetLastError();
}

}  // namespace sharq
