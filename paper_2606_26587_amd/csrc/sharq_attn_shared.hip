// Attention behind a shared prefix: one launch whose first workgroups take all
// rows' part over the prefix and whose others take the sequences' own parts.
// Neither fills the chip by itself (the prefix is a few tiles of rows, bound by
// its latencies; the own parts stream HBM), so they run side by side: in two
// launches one after the other, 64 tokens behind 8192 shared ones with 130 to 400
// of their own took 25 + 20 us, now 33; 43 x up to 10 tokens, 16 heads a
// key/value head, behind 4160 39.5, now 29.7.

#include "sharq_attn_few.hpp"
#include "sharq_attn_rows.hpp"

namespace sharq {

// Where the sequences have more rows than the kernel for few takes: prefix first as well.
template <int D, bool MX>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_attn_shared_rows(AttnArgs a, AttnSplit prefix,
                                                                          int prefix_blocks, AttnSplit own) {
  __shared__ RowsLds<D> lds;
  const int block = (int)blockIdx.x;
  if (block < prefix_blocks) attn_rows<D, MX, true>(a, block, prefix.tiles, prefix.chunk_tiles, own.chunks, lds);
  else attn_rows<D, MX, false>(a, block - prefix_blocks, own.tiles, own.chunk_tiles, 0, lds);
}

template <int D, bool MX, int NQ, int NT>
__global__ __launch_bounds__(256, 2) void k_attn_shared(AttnArgs a, AttnSplit prefix, int prefix_blocks, int chunk_tiles,
                                                        int own_chunks) {
  __shared__ union {
    RowsLds<D> rows;
    FewLds<D> few;
  } lds;
  const int block = (int)blockIdx.x;
  if (block < prefix_blocks) attn_rows<D, MX, true>(a, block, prefix.tiles, prefix.chunk_tiles, own_chunks, lds.rows);
  else attn_few<D, MX, NQ, NT>(a, block - prefix_blocks, chunk_tiles, 0, lds.few);
}

// Prompts and single tokens over an MXFP4 cache in one call, none of them split: the tiles of 128 rows first, then a
// workgroup for each sequence of few rows.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_attn_mixed(AttnArgs a, int rows_blocks, int tiles) {
  __shared__ union {
    RowsLds<D> rows;
    FewLds<D> few;
  } lds;
  const int block = (int)blockIdx.x;
  if (block < rows_blocks) attn_rows<D, true, false>(a, block, tiles, 1 << 30, 0, lds.rows);
  else attn_few<D, true, 1, 2>(a, block - rows_blocks, 1 << 30, 0, lds.few);
}

hipError_t launch_attn_mixed(const AttnArgs& a, int D, const AttnPlan& p, hipStream_t st) {
  const int first = p.own.tiles * a.c.heads;
  const dim3 g((unsigned)first + (unsigned)a.b.seqs * (unsigned)a.c.heads);
  if (D == 128) k_attn_mixed<128><<<g, 256, 0, st>>>(a, first, p.own.tiles);
  else k_attn_mixed<64><<<g, 256, 0, st>>>(a, first, p.own.tiles);
  return hipGetLastError();
}

template <int D, bool MX>
static void shared(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  constexpr int NT = MX ? 2 : 1;
  const int first = p.prefix.tiles * p.prefix.chunks * a.c.heads, ct = p.own.chunk_tiles, oc = p.own.chunks;
  const unsigned units = p.few ? (unsigned)a.b.seqs : (unsigned)p.own.tiles;
  const dim3 g((unsigned)first + (unsigned)oc * units * (unsigned)a.c.heads);
  if (p.few == 0) k_attn_shared_rows<D, MX><<<g, 256, 0, st>>>(a, p.prefix, first, p.own);
  if (p.few == 1) k_attn_shared<D, MX, 1, NT><<<g, 256, 0, st>>>(a, p.prefix, first, ct, oc);
  if constexpr (D == 64 || MX)
    if (p.few == 2) k_attn_shared<D, MX, 2, NT><<<g, 256, 0, st>>>(a, p.prefix, first, ct, oc);
  if constexpr (D == 64 && MX)
    if (p.few == 4) k_attn_shared<D, MX, 4, NT><<<g, 256, 0, st>>>(a, p.prefix, first, ct, oc);
}

hipError_t launch_attn_shared(const AttnArgs& a, int D, bool mx, const AttnPlan& p, hipStream_t st) {
  if (D == 128) mx ? shared<128, true>(a, p, st) : shared<128, false>(a, p, st);
  else mx ? shared<64, true>(a, p, st) : shared<64, false>(a, p, st);
  return hipGetLastError();
}

}  // namespace sharq
