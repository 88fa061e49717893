// Argument checks that the calls on a paged cache share.
#pragma once

#include <hip/hip_runtime.h>
#include <limits.h>

#include "../../include/sharq.h"
#include "sharq_kv.hpp"

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
  if (c->fmt != SHARQ_KV_BF16 && c->fmt != SHARQ_KV_MXFP4 && c->fmt != SHARQ_KV_FP8) return SHARQ_EINVAL;
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
  if (c->fmt != SHARQ_KV_BF16) {
    if (!c->k_scale || !c->v_scale) return SHARQ_EINVAL;
    if (c->fmt == SHARQ_KV_FP8) return SHARQ_OK;   // scales are read one by one
    if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return SHARQ_EALIGN;
  }
  return SHARQ_OK;
}

sharq::KvCacheArgs cache_args(const sharq_kv_cache* c) {
  return {static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, (int)c->pages,
          c->kv_heads, __builtin_ctz((unsigned)c->page_size)};
}

}  // namespace
