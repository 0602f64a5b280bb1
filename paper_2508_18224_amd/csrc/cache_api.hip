// C ABI of the calls over a paged cache (see include/nsa_sel.h): argument validation, workspace size, launch parameters.
#include "cache.h"

namespace nsa {
namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// 16 bytes for tensors; null only where `or_null`
bool tensor(const void* p, bool or_null = false) { return p ? aligned(p, 16) : or_null; }
bool ints(const void* p, bool or_null = false) { return p ? aligned(p, 4) : or_null; }

int check_cache_shape(const nsa_sel_cache_shape* s, bool attention) {
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

Cache make_cache(const nsa_sel_cache_shape* s, const void* k, const void* v, const float* ks, const float* vs, const int32_t* table,
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

int check_cache_pointers(const nsa_sel_cache_shape* s, const void* k, const void* v, const float* ks, const float* vs,
                         const int32_t* table, const int32_t* kv_len, const int32_t* cu) {
  if (!ints(kv_len) || !ints(cu, true) || !ints(table, s->max_pages == 0)) return NSA_SEL_EINVAL;
  if (!cu && s->nseq != s->n_tokens) return NSA_SEL_EINVAL;
  const bool none = s->n_pages == 0;
  if (!tensor(k, none) || !tensor(v, none)) return NSA_SEL_EINVAL;
  if (s->dtype == NSA_SEL_CACHE_E4M3 && (!ints(ks, none) || !ints(vs, none))) return NSA_SEL_EINVAL;
  return NSA_SEL_OK;
}

// How the attention is cut: new tokens a workgroup takes together, and workgroups that share a row's keys.
struct Cut {
  int group, splits;
};
Cut cut_of(const nsa_sel_cache_shape* s) {
  Cut c;
  const int g = s->hq / s->hkv;
  const int64_t each = s->nseq > 0 ? (s->n_tokens + (int64_t)s->nseq - 1) / s->nseq : 1;  // new tokens of a sequence, in the mean
  const int64_t most = 16 / g;
  c.group = s->topk > 0 ? 1 : (int)(each < most ? (each > 1 ? each : 1) : most);
  const int64_t rows = (s->n_tokens + c.group - 1) / c.group * (int64_t)s->hkv;
  int64_t keys = (int64_t)s->max_pages * s->page;
  if (s->topk > 0 && (int64_t)s->topk * s->block < keys) keys = (int64_t)s->topk * s->block;
  if (s->window > 0 && (int64_t)s->window + c.group < keys) keys = (int64_t)s->window + c.group;
  const int64_t pieces = (keys + kAttendPiece - 1) / kAttendPiece, target = s->topk > 0 || s->window > 0 ? 512 : 2048;
  int64_t n = rows > 0 ? (target + rows - 1) / rows : 1;
  const int64_t cap = (pieces + kAttendWaves - 1) / kAttendWaves;  // a piece a wavefront
  if (n > cap) n = cap;
  c.splits = (int)(n < 1 ? 1 : n > 128 ? 128 : n);
  return c;
}
size_t part_bytes(const nsa_sel_cache_shape* s, const Cut& c) { return (size_t)s->n_tokens * s->hq * c.splits * kD * 4; }
size_t cache_ws_bytes(const nsa_sel_cache_shape* s, const Cut& c) {
  return c.splits == 1 ? 0 : part_bytes(s, c) + (size_t)s->n_tokens * s->hq * c.splits * 8;
}

}  // namespace
}  // namespace nsa

using namespace nsa;

extern "C" {

int nsa_sel_cache_append(const nsa_sel_cache_shape* shape, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                         const void* V, int64_t v_stride, const int32_t* cu_seqlens, const int32_t* kv_len,
                         const int32_t* table, const double* inv_freq, int32_t rot, int32_t interleaved, void* k_pages,
                         void* v_pages, float* k_scale, float* v_scale, void* Q_out, void* K_out, void* stream) {
  int rc = check_cache_shape(shape, false);
  if (rc) return rc;
  if (rot < 0 || rot > kD || (rot & 15) != 0) return NSA_SEL_EINVAL;
  if (shape->n_tokens == 0) return NSA_SEL_OK;
  rc = check_cache_pointers(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  if (rc) return rc;
  if (!tensor(K) || !tensor(V) || !tensor(Q, true) || !tensor(Q_out, true) || !tensor(K_out, true)) return NSA_SEL_EINVAL;
  if ((Q == nullptr) != (Q_out == nullptr) || (rot > 0 && (!inv_freq || !aligned(inv_freq, 8)))) return NSA_SEL_EINVAL;
  const int64_t kv = (int64_t)shape->hkv * kD, q = (int64_t)shape->hq * kD;
  if (k_stride < kv || v_stride < kv || (k_stride & 7) || (v_stride & 7) || (Q && (q_stride < q || (q_stride & 7)))) return NSA_SEL_EINVAL;
  if ((Q && Q_out == Q && q_stride != q) || (K_out == K && k_stride != kv)) return NSA_SEL_EINVAL;
  const int64_t units = cu_seqlens ? shape->n_tokens / shape->page + 2 * (int64_t)shape->nseq : shape->nseq;
  if (2 * units * shape->hkv + shape->n_tokens >= ((int64_t)1 << 31)) return NSA_SEL_EUNSUPPORTED;  // workgroups
  const Cache C = make_cache(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  return launch_cache_append(C, shape->dtype == NSA_SEL_CACHE_E4M3, Q, q_stride, K, k_stride, V, v_stride, inv_freq, rot,
                             interleaved != 0, Q_out, K_out, (hipStream_t)stream) == hipSuccess
             ? NSA_SEL_OK
             : NSA_SEL_EHIP;
}

int nsa_sel_cache_workspace_bytes(const nsa_sel_cache_shape* shape, size_t* bytes) {
  int rc = check_cache_shape(shape, true);
  if (rc) return rc;
  if (bytes) *bytes = cache_ws_bytes(shape, cut_of(shape));
  return NSA_SEL_OK;
}

int nsa_sel_cache_attention(const nsa_sel_cache_shape* shape, const void* Q, const int32_t* idx, const int32_t* cu_seqlens,
                            const int32_t* kv_len, const int32_t* table, const void* k_pages, const void* v_pages,
                            const float* k_scale, const float* v_scale, const float* gate, const void* O_acc, void* O,
                            float* LSE, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_cache_shape(shape, true);
  if (rc) return rc;
  if (shape->n_tokens == 0) return NSA_SEL_OK;
  rc = check_cache_pointers(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  if (rc) return rc;
  if (!tensor(Q) || !tensor(O) || !ints(LSE) || !tensor(O_acc, true) || !ints(gate, true)) return NSA_SEL_EINVAL;
  if ((shape->topk > 0) != (idx != nullptr) || !ints(idx, true) || (O_acc && !gate) || O == Q) return NSA_SEL_EINVAL;
  const Cut c = cut_of(shape);
  const size_t need = cache_ws_bytes(shape, c);
  if (need > 0 && !tensor(ws)) return NSA_SEL_EINVAL;
  if (ws_bytes < need) return NSA_SEL_EWORKSPACE;
  const int64_t groups = c.group > 1 ? shape->n_tokens / c.group + (int64_t)shape->nseq : shape->n_tokens;
  if (groups * shape->hkv * c.splits >= ((int64_t)1 << 31)) return NSA_SEL_EUNSUPPORTED;  // workgroups
  CacheAttend A;
  A.Q = Q;
  A.idx = idx;
  A.block = shape->topk > 0 ? shape->block : kBlock;
  A.topk = shape->topk;
  A.window = shape->window;
  A.scale = shape->scale > 0.f ? shape->scale : 0.08838834764831845f;  // 1/sqrt(128)
  A.gate = gate;
  A.o_acc = O_acc;
  A.O = O;
  A.LSE = LSE;
  A.group = c.group;
  A.splits = c.splits;
  A.part = (float*)ws;
  A.part_ml = (float2*)((char*)ws + part_bytes(shape, c));
  const Cache C = make_cache(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  return launch_cache_attend(C, shape->dtype == NSA_SEL_CACHE_E4M3, A, (hipStream_t)stream) == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP;
}

}  // extern "C"
