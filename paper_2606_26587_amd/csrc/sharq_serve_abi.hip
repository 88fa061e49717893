// C ABI of the calls around the paged cache: argument validation and dispatch.
// The entry points and their contracts are declared in include/sharq.h.

#include <limits.h>

#include "../../include/sharq.h"
#include "sharq_kv_check.hpp"
#include "sharq_serve.hpp"

namespace sharq {
hipError_t launch_kv_assign(const AssignArgs& a, hipStream_t st);
hipError_t launch_beam_select(const BeamArgs& a, int64_t groups, int dtype, hipStream_t st);
hipError_t launch_beam_reorder(const ReorderArgs& a, int64_t groups, hipStream_t st);
hipError_t launch_kv_copy(const KvCacheArgs& c, const int32_t* copies, int64_t n, int D, int fmt, hipStream_t st);
}  // namespace sharq

namespace {

using namespace sharq;

constexpr int64_t kMaxColumns = (int64_t)1 << 30;   // of all sequences: pages given out are counted in 32 bits
constexpr int64_t kMaxBeamRows = (int64_t)1 << 20;
constexpr int64_t kMaxCandidates = (int64_t)1 << 30;   // of a group

bool page_size_ok(int64_t p) { return p >= 1 && (p & (p - 1)) == 0; }

sharq_status check_requests(const sharq_kv_requests* r) {
  if (!r || r->seqs < 0 || r->rows < 0 || r->rows > INT_MAX || r->max_len < 0 || r->ld_table < 0 ||
      !page_size_ok(r->page_size))
    return SHARQ_EINVAL;
  if (r->page_size < 16 || r->page_size > 1024 || r->seqs > kMaxSeqs || r->max_len > kMaxLen) return SHARQ_EUNSUPPORTED;
  const int64_t cols = (r->max_len + r->page_size - 1) / r->page_size;
  if (r->seqs > 0 && cols > r->ld_table) return SHARQ_EINVAL;
  if (r->seqs * cols > kMaxColumns) return SHARQ_EUNSUPPORTED;
  return SHARQ_OK;
}

sharq_status check_beams(int64_t groups, int64_t beams) {
  if (groups < 0 || beams < 1) return SHARQ_EINVAL;
  if (beams > kMaxBeams || groups > kMaxBeamRows / beams) return SHARQ_EUNSUPPORTED;
  return SHARQ_OK;
}

sharq_status check_choice(int64_t groups, int64_t beams, int64_t vocab) {
  const sharq_status s = check_beams(groups, beams);
  if (s != SHARQ_OK) return s;
  if (vocab < 1) return SHARQ_EINVAL;
  return vocab > kMaxCandidates / beams ? SHARQ_EUNSUPPORTED : SHARQ_OK;
}

}  // namespace

extern "C" {

size_t sharq_kv_assign_workspace_bytes(const sharq_kv_requests* r) {
  return check_requests(r) == SHARQ_OK ? (size_t)assign_workspace(r->seqs) : 0;
}

sharq_status sharq_kv_assign(const sharq_kv_pool* pool, const sharq_kv_requests* r, void* workspace,
                             size_t workspace_bytes, void* stream) {
  const sharq_status s = check_requests(r);
  if (s != SHARQ_OK) return s;
  if (!pool || pool->pages < 0 || !pool->count || !pool->count_out || !r->row_offsets) return SHARQ_EINVAL;
  if (pool->pages > INT_MAX / r->page_size) return SHARQ_EUNSUPPORTED;   // slots are counted in 32 bits
  if (pool->pages > 0 && !pool->free_pages) return SHARQ_EINVAL;
  if (r->seqs > 0 && (!r->keep || !r->add || !r->held || !r->held_out || !r->lens ||
                      (!r->page_table && r->max_len > 0)))
    return SHARQ_EINVAL;
  for (const void* p : {(const void*)pool->free_pages, (const void*)pool->count, (const void*)pool->count_out,
                        (const void*)r->keep, (const void*)r->add, (const void*)r->held, (const void*)r->held_out,
                        (const void*)r->row_offsets, (const void*)r->lens, (const void*)r->page_table,
                        (const void*)r->own_table, (const void*)r->row_seq, (const void*)r->positions,
                        (const void*)r->slots, (const void*)r->missing, (const void*)workspace})
    if (!aligned(p, 4)) return SHARQ_EALIGN;
  if (r->seqs > 0 && (!workspace || workspace_bytes < (size_t)assign_workspace(r->seqs))) return SHARQ_EINVAL;
  const AssignArgs a{pool->free_pages, pool->count, pool->count_out, r->missing, r->keep, r->add, r->held, r->held_out,
                     r->row_offsets, r->lens, r->page_table, r->own_table, r->row_seq, r->positions, r->slots,
                     static_cast<int32_t*>(workspace), r->ld_table, (int)pool->pages, (int)r->seqs, (int)r->rows,
                     (int)r->max_len, (int)((r->max_len + r->page_size - 1) / r->page_size),
                     __builtin_ctz((unsigned)r->page_size)};
  return hip_status(launch_kv_assign(a, reinterpret_cast<hipStream_t>(stream)));
}

size_t sharq_beam_workspace_bytes(int64_t groups, int64_t beams, int64_t vocab) {
  if (check_choice(groups, beams, vocab) != SHARQ_OK) return 0;
  return (size_t)beam_workspace(groups * beams, beams, vocab);
}

sharq_status sharq_beam_select(const void* logits, sharq_dtype dtype, int64_t ld, int64_t groups, int64_t beams,
                               int64_t vocab, const float* scores, const uint8_t* done, int32_t eos, float* scores_out,
                               int32_t* parents, int32_t* tokens, uint8_t* done_out, void* workspace,
                               size_t workspace_bytes, void* stream) {
  const sharq_status s = check_choice(groups, beams, vocab);
  if (s != SHARQ_OK) return s;
  if (ld < vocab || eos < -1 || eos >= vocab || (done && eos < 0) || (done == nullptr) != (done_out == nullptr))
    return SHARQ_EINVAL;
  if (dtype != SHARQ_BF16 && dtype != SHARQ_F16 && dtype != SHARQ_F32) return SHARQ_EINVAL;
  if (groups == 0) return SHARQ_OK;
  if (!logits || !scores || !scores_out || !parents || !tokens || !workspace) return SHARQ_EINVAL;
  if (!aligned(logits, dtype == SHARQ_F32 ? 4 : 2) || !aligned(scores, 4) || !aligned(scores_out, 4) ||
      !aligned(parents, 4) || !aligned(tokens, 4) || !aligned(workspace, 8))
    return SHARQ_EALIGN;
  if (workspace_bytes < (size_t)beam_workspace(groups * beams, beams, vocab)) return SHARQ_EINVAL;
  const BeamSplit split = beam_split(groups * beams, beams, vocab);
  uint64_t* const lists = static_cast<uint64_t*>(workspace);
  const BeamArgs a{logits, ld, scores, done, scores_out, parents, tokens, done_out, lists,
                   reinterpret_cast<BeamPart*>(lists + groups * beams * split.chunks * beams), (int)beams, (int)vocab,
                   eos, split.chunks, split.tiles};
  return hip_status(launch_beam_select(a, groups, dtype, reinterpret_cast<hipStream_t>(stream)));
}

sharq_status sharq_beam_reorder(int64_t groups, int64_t beams, const int32_t* parents, const int32_t* lens,
                                int32_t page_size, const int32_t* table, int64_t ldt, int32_t* table_out, int64_t ldto,
                                int64_t cols, int32_t* copies, const int32_t* tokens, const int32_t* ids, int64_t ldi,
                                int32_t* ids_out, int64_t ldio, int64_t id_cols, void* stream) {
  const sharq_status s = check_beams(groups, beams);
  if (s != SHARQ_OK) return s;
  if (!page_size_ok(page_size) || cols < 0 || id_cols < 0) return SHARQ_EINVAL;
  if (page_size < 16 || page_size > 1024 || cols > kMaxLen || id_cols > kMaxLen) return SHARQ_EUNSUPPORTED;
  if ((table == nullptr) != (table_out == nullptr) || (copies && !table) || (ids == nullptr) != (ids_out == nullptr) ||
      (ids && !tokens))
    return SHARQ_EINVAL;
  if ((table && (ldt < cols || ldto < cols || !copies)) || (ids && (ldi < id_cols || ldio < id_cols)))
    return SHARQ_EINVAL;
  if ((table && table == table_out && ldt != ldto) || (ids && ids == ids_out && ldi != ldio)) return SHARQ_EINVAL;
  for (const void* p : {(const void*)parents, (const void*)lens, (const void*)table, (const void*)table_out,
                        (const void*)copies, (const void*)tokens, (const void*)ids, (const void*)ids_out})
    if (!aligned(p, 4)) return SHARQ_EALIGN;
  if (groups == 0 || (!table && !ids)) return SHARQ_OK;
  if (!parents || !lens) return SHARQ_EINVAL;
  const int64_t units = (table ? reorder_units(cols > 0 ? cols : 1) : 0) + (ids ? reorder_units(id_cols) : 0);
  if (units == 0) return SHARQ_OK;   // token ids without columns
  if (!kv_launches(groups * ((units + 3) / 4), 256)) return SHARQ_EUNSUPPORTED;
  const ReorderArgs a{parents, lens, tokens, table, table_out, ldt, ldto, ids, ids_out, ldi, ldio, copies, (int)beams,
                      (int)cols, (int)id_cols, __builtin_ctz((unsigned)page_size)};
  return hip_status(launch_beam_reorder(a, groups, reinterpret_cast<hipStream_t>(stream)));
}

sharq_status sharq_kv_copy(const sharq_kv_cache* cache, const int32_t* copies, int64_t n, void* stream) {
  const sharq_status s = check_cache(cache);
  if (s != SHARQ_OK) return s;
  if (n < 0) return SHARQ_EINVAL;
  if (n == 0 || cache->pages == 0) return SHARQ_OK;
  if (!copies) return SHARQ_EINVAL;
  if (!aligned(copies, 4)) return SHARQ_EALIGN;
  const int64_t per = cache->kv_heads * copy_parts(cache->page_size, cache->head_dim, cache->fmt);
  if (n > kMaxHeadRows || !kv_launches(n * per, 256)) return SHARQ_EUNSUPPORTED;
  return hip_status(launch_kv_copy(cache_args(cache), copies, n, cache->head_dim, cache->fmt,
                                   reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
