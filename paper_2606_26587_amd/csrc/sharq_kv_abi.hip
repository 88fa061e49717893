// C ABI of the paged key/value cache and its attention: argument validation and
// dispatch.  The entry points and their contracts are declared in
// include/sharq.h.

#include <limits.h>

#include "../../include/sharq.h"
#include "sharq_device.hpp"
#include "sharq_kv.hpp"

namespace sharq {
hipError_t launch_kv_append(const uint16_t* q, const uint16_t* k, const uint16_t* v, int64_t ldq, int64_t ldk,
                            int64_t ldv, int q_heads, uint16_t* qo, int64_t ldqo, const float* cos, const float* sin,
                            int angles, const int32_t* pos, uint32_t rule_bias, const KvBatchArgs& b,
                            const KvCacheArgs& c, int D, bool mx, hipStream_t st);
hipError_t launch_kv_read(uint16_t* ko, int64_t ldk, uint16_t* vo, int64_t ldv, const KvBatchArgs& b,
                          const KvCacheArgs& c, int D, bool mx, hipStream_t st);
hipError_t launch_attention(const uint16_t* q, int64_t ldq, uint16_t* o, int64_t ldo, float* lse,
                            const KvBatchArgs& b, const KvCacheArgs& c, const AttnPlan& plan,
                            const int32_t* prefix_table, int prefix_len, int q_heads, int D, bool mx, int window,
                            int sinks, float scale, void* ws, hipStream_t st);
}  // namespace sharq

namespace {

constexpr int64_t kMaxLen = (int64_t)1 << 30;
constexpr int64_t kMaxSeqs = (int64_t)1 << 16;
constexpr int64_t kMaxHeads = 1024;
constexpr int64_t kMaxGroup = 128;
constexpr float kMinScale = 0x1p-100f, kMaxScale = 0x1p100f;   // scale times log2 e and times a maximum's start stay normal
constexpr int64_t kMaxHeadRows = (int64_t)1 << 26;   // rows times heads of a call: row and head numbers fit 27 bits

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool row_aligned(const void* p, int64_t ld) { return aligned(p, 16) && (ld * 2) % 16 == 0; }
sharq_status hip_status(hipError_t e) { return e == hipSuccess ? SHARQ_OK : SHARQ_EHIP; }

// Sizes and format of a cache.
sharq_status check_sizes(const sharq_kv_cache* c) {
  if (!c) return SHARQ_EINVAL;
  if (c->fmt != SHARQ_KV_BF16 && c->fmt != SHARQ_KV_MXFP4) return SHARQ_EINVAL;
  if (c->pages < 0 || c->kv_heads < 1 || c->page_size < 1 || (c->page_size & (c->page_size - 1)) != 0 ||
      c->head_dim < 1)
    return SHARQ_EINVAL;
  if (c->scale_rule != SHARQ_SCALE_FLOOR && c->scale_rule != SHARQ_SCALE_CEIL) return SHARQ_EINVAL;
  if (c->page_size < 16 || c->page_size > 1024 || c->kv_heads > kMaxHeads) return SHARQ_EUNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return SHARQ_EUNSUPPORTED;
  if (c->pages > INT_MAX / ((int64_t)c->kv_heads * c->page_size)) return SHARQ_EUNSUPPORTED;
  return SHARQ_OK;
}

sharq_status check_cache(const sharq_kv_cache* c) {
  const sharq_status s = check_sizes(c);
  if (s != SHARQ_OK || c->pages == 0) return s;   // an empty pool is never dereferenced
  if (!c->k || !c->v) return SHARQ_EINVAL;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return SHARQ_EALIGN;
  if (c->fmt == SHARQ_KV_MXFP4) {
    if (!c->k_scale || !c->v_scale) return SHARQ_EINVAL;
    if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return SHARQ_EALIGN;
  }
  return SHARQ_OK;
}

// arrays: whether the device arrays must be there (they need not for sizing).
sharq_status check_batch(const sharq_kv_batch* b, const sharq_kv_cache* c, bool arrays) {
  if (!b) return SHARQ_EINVAL;
  if (b->seqs < 0 || b->rows < 0 || b->rows > INT_MAX || b->max_rows < 0 || b->max_len < 0 || b->ld_table < 0)
    return SHARQ_EINVAL;
  if (b->seqs > kMaxSeqs || b->max_len > kMaxLen) return SHARQ_EUNSUPPORTED;
  if (b->seqs == 0 || b->rows == 0) return SHARQ_OK;   // nothing is launched
  if ((b->max_len + c->page_size - 1) / c->page_size > b->ld_table) return SHARQ_EINVAL;
  if (!arrays) return SHARQ_OK;
  if (!b->row_offsets || !b->lens || (!b->page_table && b->max_len > 0)) return SHARQ_EINVAL;
  if (!aligned(b->row_offsets, 4) || !aligned(b->lens, 4) || !aligned(b->page_table, 4)) return SHARQ_EALIGN;
  return SHARQ_OK;
}

sharq::KvCacheArgs cache_args(const sharq_kv_cache* c) {
  return {static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, (int)c->pages,
          c->kv_heads, __builtin_ctz((unsigned)c->page_size)};
}

sharq::KvBatchArgs batch_args(const sharq_kv_batch* b, int64_t rows) {
  return {b->row_offsets, b->lens, b->page_table, b->ld_table, (int)b->seqs, (int)rows, (int)b->max_len};
}

// Rows that sequences can own: those behind are padding, which the attention keeps no partial results of.
int64_t owned_rows(const sharq_kv_batch* b) {
  return b->max_rows < b->rows && b->seqs * b->max_rows < b->rows ? b->seqs * b->max_rows : b->rows;
}

sharq_status check_attn(const sharq_attn* t, const sharq_kv_cache* c, const sharq_kv_batch* b, int64_t q_heads,
                        bool arrays) {
  if (!t || q_heads < 1 || q_heads % c->kv_heads != 0) return SHARQ_EINVAL;
  if (q_heads / c->kv_heads > kMaxGroup || b->rows * q_heads > kMaxHeadRows || b->seqs * c->kv_heads > 1 << 22)
    return SHARQ_EUNSUPPORTED;
  if (!(t->scale > 0.0f) || __builtin_isinf(t->scale) || t->window < 0 || t->sinks < 0) return SHARQ_EINVAL;
  if (t->prefix_len < 0 || t->prefix_len > b->max_len || t->prefix_len % c->page_size != 0) return SHARQ_EINVAL;
  if (t->scale < kMinScale || t->scale > kMaxScale) return SHARQ_EUNSUPPORTED;
  if (!arrays) return SHARQ_OK;
  if (t->prefix_len > 0 && !t->prefix_table) return SHARQ_EINVAL;
  if (!aligned(t->prefix_table, 4)) return SHARQ_EALIGN;
  return SHARQ_OK;
}

int attn_window(const sharq_attn* t) { return t->window == 0 || t->window > INT_MAX ? INT_MAX : (int)t->window; }
int attn_sinks(const sharq_attn* t) { return t->sinks > INT_MAX ? INT_MAX : (int)t->sinks; }

sharq::AttnPlan plan_of(const sharq_kv_cache* c, const sharq_kv_batch* b, const sharq_attn* t, int64_t q_heads) {
  return sharq::attn_plan(b->seqs, owned_rows(b), b->max_rows, b->max_len, c->kv_heads, (int)(q_heads / c->kv_heads),
                          c->head_dim, c->fmt == SHARQ_KV_MXFP4, attn_window(t), attn_sinks(t), t->prefix_len);
}

}  // namespace

extern "C" {

size_t sharq_kv_buffer_bytes(const sharq_kv_cache* c, int32_t which) {
  if (check_sizes(c) != SHARQ_OK || which < 0 || which > 3) return 0;
  const size_t values = (size_t)c->pages * (size_t)c->kv_heads * (size_t)c->page_size * (size_t)c->head_dim;
  if (which < 2) return c->fmt == SHARQ_KV_BF16 ? values * 2 : values / 2;
  return c->fmt == SHARQ_KV_BF16 ? 0 : values / 32;
}

sharq_status sharq_kv_append(const void* Q, const void* K, const void* V, sharq_dtype xdt, int64_t q_heads,
                             int64_t ldq, int64_t ldk, int64_t ldv, const float* cos, const float* sin, int64_t angles,
                             const int32_t* positions, const sharq_kv_cache* cache, const sharq_kv_batch* batch,
                             void* Q_out, int64_t ldqo, void* stream) {
  sharq_status s = check_cache(cache);
  if (s != SHARQ_OK) return s;
  s = check_batch(batch, cache, true);
  if (s != SHARQ_OK) return s;
  const int64_t D = cache->head_dim, wk = cache->kv_heads * D;
  if (q_heads < 0 || ldk < wk || ldv < wk || (q_heads > 0 && (ldq < q_heads * D || ldqo < q_heads * D)))
    return SHARQ_EINVAL;
  if ((cos == nullptr) != (sin == nullptr) || (cos && (angles < 0 || angles > INT_MAX)) || (positions && !cos))
    return SHARQ_EINVAL;
  if (xdt != SHARQ_BF16 || q_heads > kMaxHeads || batch->rows * (q_heads + 2 * cache->kv_heads) > kMaxHeadRows)
    return SHARQ_EUNSUPPORTED;
  if (batch->rows == 0 || batch->seqs == 0) return SHARQ_OK;
  if (!K || !V || (q_heads > 0 && (!Q || !Q_out))) return SHARQ_EINVAL;
  if (!row_aligned(K, ldk) || !row_aligned(V, ldv) || !aligned(cos, 16) || !aligned(sin, 16) ||
      !aligned(positions, 4) || (q_heads > 0 && (!row_aligned(Q, ldq) || !row_aligned(Q_out, ldqo))))
    return SHARQ_EALIGN;
  if (batch->max_len == 0) return SHARQ_OK;   // no row has a position
  if (!sharq::kv_launches(batch->rows * sharq::kv_append_parts((int)q_heads, cache->kv_heads, (int)D),
                          sharq::kAppendThreads))
    return SHARQ_EUNSUPPORTED;
  return hip_status(sharq::launch_kv_append(
      static_cast<const uint16_t*>(Q), static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V), ldq, ldk, ldv,
      (int)q_heads, static_cast<uint16_t*>(Q_out), ldqo, cos, sin, (int)angles, positions,
      cache->scale_rule == SHARQ_SCALE_CEIL ? sharq::kE8Ceil : sharq::kE8Floor, batch_args(batch, batch->rows),
      cache_args(cache), (int)D, cache->fmt == SHARQ_KV_MXFP4, reinterpret_cast<hipStream_t>(stream)));
}

sharq_status sharq_kv_read(const sharq_kv_cache* cache, const sharq_kv_batch* batch, void* K, int64_t ldk, void* V,
                           int64_t ldv, sharq_dtype ydt, void* stream) {
  sharq_status s = check_cache(cache);
  if (s != SHARQ_OK) return s;
  s = check_batch(batch, cache, true);
  if (s != SHARQ_OK) return s;
  const int64_t wk = (int64_t)cache->kv_heads * cache->head_dim;
  if (ldk < wk || ldv < wk) return SHARQ_EINVAL;
  if (ydt != SHARQ_BF16 || batch->rows * 2 * cache->kv_heads > kMaxHeadRows) return SHARQ_EUNSUPPORTED;
  if (batch->rows == 0 || batch->seqs == 0) return SHARQ_OK;
  if (!K || !V) return SHARQ_EINVAL;
  if (!row_aligned(K, ldk) || !row_aligned(V, ldv)) return SHARQ_EALIGN;
  if (!sharq::kv_launches(batch->rows * sharq::kv_read_parts(cache->kv_heads, cache->head_dim), sharq::kReadThreads))
    return SHARQ_EUNSUPPORTED;
  return hip_status(sharq::launch_kv_read(static_cast<uint16_t*>(K), ldk, static_cast<uint16_t*>(V), ldv,
                                          batch_args(batch, batch->rows), cache_args(cache), cache->head_dim,
                                          cache->fmt == SHARQ_KV_MXFP4, reinterpret_cast<hipStream_t>(stream)));
}

size_t sharq_attention_workspace_bytes(const sharq_kv_cache* cache, const sharq_kv_batch* batch,
                                       const sharq_attn* attn, int64_t q_heads) {
  if (check_sizes(cache) != SHARQ_OK || check_batch(batch, cache, false) != SHARQ_OK ||
      check_attn(attn, cache, batch, q_heads, false) != SHARQ_OK)
    return 0;
  if (batch->rows == 0 || batch->seqs == 0 || batch->max_rows == 0) return 0;
  return (size_t)sharq::attn_workspace(owned_rows(batch) * q_heads, plan_of(cache, batch, attn, q_heads).slots,
                                       cache->head_dim);
}

sharq_status sharq_attention(const void* Q, sharq_dtype xdt, int64_t q_heads, int64_t ldq,
                             const sharq_kv_cache* cache, const sharq_kv_batch* batch, const sharq_attn* attn, void* O,
                             int64_t ldo, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  sharq_status s = check_cache(cache);
  if (s != SHARQ_OK) return s;
  s = check_batch(batch, cache, true);
  if (s != SHARQ_OK) return s;
  s = check_attn(attn, cache, batch, q_heads, true);
  if (s != SHARQ_OK) return s;
  const int64_t D = cache->head_dim;
  if (ldq < q_heads * D || ldo < q_heads * D) return SHARQ_EINVAL;
  if (xdt != SHARQ_BF16) return SHARQ_EUNSUPPORTED;
  if (batch->rows == 0 || batch->seqs == 0 || batch->max_rows == 0) return SHARQ_OK;
  if (!Q || !O) return SHARQ_EINVAL;
  if (!row_aligned(Q, ldq) || !row_aligned(O, ldo) || !aligned(lse, 4) || !aligned(workspace, 16)) return SHARQ_EALIGN;
  const sharq::AttnPlan plan = plan_of(cache, batch, attn, q_heads);
  const size_t need = (size_t)sharq::attn_workspace(owned_rows(batch) * q_heads, plan.slots, (int)D);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SHARQ_EINVAL;
  if (O == Q) return SHARQ_EINVAL;   // several workgroups read a row's queries
  return hip_status(sharq::launch_attention(
      static_cast<const uint16_t*>(Q), ldq, static_cast<uint16_t*>(O), ldo, lse, batch_args(batch, owned_rows(batch)),
      cache_args(cache), plan, attn->prefix_table, (int)attn->prefix_len, (int)q_heads, (int)D,
      cache->fmt == SHARQ_KV_MXFP4, attn_window(attn), attn_sinks(attn), attn->scale, workspace, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
