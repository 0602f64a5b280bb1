// Host checks that the calls over a paged cache share: sizes, pointers, and the description of the cache that their kernels take.
#pragma once
#include "cache.h"

namespace nsa {

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// 16 bytes for tensors; null only where `or_null`
inline bool tensor(const void* p, bool or_null = false) { return p ? aligned(p, 16) : or_null; }
inline bool ints(const void* p, bool or_null = false) { return p ? aligned(p, 4) : or_null; }

inline int check_sizes(const nsa_sel_cache_shape* s, bool attention) {
  if (!s) return NSA_SEL_EINVAL;
  if (s->n_tokens < 0 || s->nseq < 0 || (s->nseq == 0 && s->n_tokens > 0) || s->hq < 1 || s->hkv < 1 || s->n_pages < 0 || s->max_pages < 0)
    return NSA_SEL_EINVAL;
  if (s->hq % s->hkv != 0 || s->hq / s->hkv > 8) return NSA_SEL_EINVAL;
  if (s->dtype != NSA_SEL_CACHE_BF16 && s->dtype != NSA_SEL_CACHE_E4M3) return NSA_SEL_EINVAL;
  if (attention && s->window < 0) return NSA_SEL_EINVAL;
  if (s->d != kD || s->page < 16 || s->page > 256 || (s->page & (s->page - 1)) != 0) return NSA_SEL_EUNSUPPORTED;
  if ((int64_t)s->max_pages * s->page > (1 << 30)) return NSA_SEL_EUNSUPPORTED;  // places are 32-bit numbers
  if (s->nseq > (1 << 24) || (int64_t)s->n_tokens * s->hq >= ((int64_t)1 << 31)) return NSA_SEL_EUNSUPPORTED;
  if (attention) {
    if (s->topk < 0 || s->topk > kMaxTopk) return NSA_SEL_EUNSUPPORTED;
    if (s->topk > 0 && s->block != kBlock && s->block != 2 * kBlock) return NSA_SEL_EUNSUPPORTED;
  }
  return NSA_SEL_OK;
}

inline Cache make_cache(const nsa_sel_cache_shape* s, const void* k, const void* v, const float* ks, const float* vs, const int32_t* table,
                 const int32_t* kv_len, const int32_t* cu) {
  Cache C;
  C.k = (char*)const_cast<void*>(k);
  C.v = (char*)const_cast<void*>(v);
  C.ks = const_cast<float*>(ks);
  C.vs = const_cast<float*>(vs);
  C.table = table;
  C.kv_len = kv_len;
  C.cu = cu;
  C.T = s->n_tokens;
  C.nseq = s->nseq;
  C.hq = s->hq;
  C.hkv = s->hkv;
  C.g = s->hq / s->hkv;
  C.n_pages = s->n_pages;
  C.max_pages = s->max_pages;
  C.page_log2 = __builtin_ctz((unsigned)s->page);
  return C;
}

inline int check_cache_pointers(const nsa_sel_cache_shape* s, const void* k, const void* v, const float* ks, const float* vs,
                         const int32_t* table, const int32_t* kv_len, const int32_t* cu) {
  if (!ints(kv_len) || !ints(cu, true) || !ints(table, s->max_pages == 0)) return NSA_SEL_EINVAL;
  if (!cu && s->nseq != s->n_tokens) return NSA_SEL_EINVAL;
  const bool none = s->n_pages == 0;
  if (!tensor(k, none) || !tensor(v, none)) return NSA_SEL_EINVAL;
  if (s->dtype == NSA_SEL_CACHE_E4M3 && (!ints(ks, none) || !ints(vs, none))) return NSA_SEL_EINVAL;
  return NSA_SEL_OK;
}

// Lengths below this one are this one: places that follow from them are negative all the same, and no sum leaves 32 bits.
constexpr int kLeastLength = -(1 << 30);

// The first place that a window shows to the token at `place`, 0 or more, for every place and window: the difference of those far apart is not formed.
constexpr int32_t window_start(int32_t place, int32_t window) { return place >= window ? place + 1 - window : 0; }
static_assert(window_start(INT32_MIN, INT32_MAX) == 0 && window_start(kLeastLength - (1 << 20), (1 << 30) - 1) == 0);
static_assert(window_start(INT32_MAX - 1, 1) == INT32_MAX - 1 && window_start(5, 6) == 0 && window_start(6, 6) == 1 && window_start(7, 6) == 2);

// No place is as far back as 2^30 of another: a window that long is none, and the kernels' sums of one with a place from -2^30 on stay in 32 bits.
inline int32_t window_of(const nsa_sel_cache_shape* s) { return s->window < (1 << 30) ? s->window : 0; }

}  // namespace nsa
