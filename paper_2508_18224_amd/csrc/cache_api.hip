// C ABI of the calls over a paged cache (see include/nsa_sel.h): argument validation, workspace size, launch parameters.
#include "cache.h"

namespace nsa {
namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// 16 bytes for tensors; null only where `or_null`
bool tensor(const void* p, bool or_null = false) { return p ? aligned(p, 16) : or_null; }
bool ints(const void* p, bool or_null = false) { return p ? aligned(p, 4) : or_null; }

int check_sizes(const nsa_sel_cache_shape* s, bool attention) {
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

// No place is as far back as 2^30 of another: a window that long is none, and the kernels' sums with one stay in 32 bits.
int32_t window_of(const nsa_sel_cache_shape* s) { return s->window < (1 << 30) ? s->window : 0; }

// How the attention is cut (see launch_cache_attend).
struct Cut {
  int group;           // new tokens of a sequence that a workgroup takes together
  int splits, chunk, even;
  bool streaming;
  int64_t slots;       // of parts; 0 where every row is one workgroup's
  int64_t workgroups;
};
Cut cut_of(const nsa_sel_cache_shape* s) {
  Cut c;
  const int g = s->hq / s->hkv;
  const int64_t each = s->nseq > 0 ? (s->n_tokens + (int64_t)s->nseq - 1) / s->nseq : 1;  // new tokens of a sequence, in the mean
  const int64_t most = 16 / g;
  c.group = s->topk > 0 ? 1 : (int)(each < most ? (each > 1 ? each : 1) : most);
  const int64_t rows = ((int64_t)s->n_tokens + c.group - 1) / c.group * s->hkv;
  // Upper bound of the pieces of a row (the kernel finds out how many there are, by the lengths and the kept blocks).  Lengths are the device's: without a
  // selection or a window all the host has is the table's width, and the rules below were measured on tables that fit their sequences.  Where the table is much
  // wider, short sequences are cut as long ones are (16 of 1024 in a table of 131072 places 14.6 -> 17.0 us, two of 4096 12.9 -> 13.5).
  const int64_t limit = (int64_t)s->max_pages * s->page, window = window_of(s);
  int64_t pieces = (limit + kAttendPiece - 1) / kAttendPiece;
  if (s->topk > 0) {
    int64_t blocks = (limit + s->block - 1) / s->block;
    if (blocks > s->topk) blocks = s->topk;
    if (window > 0 && blocks > window / s->block + 2) blocks = window / s->block + 2;
    pieces = blocks * (s->block / kAttendPiece);
  } else if (window > 0 && pieces > (window + c.group) / kAttendPiece + 2) {
    pieces = (window + c.group) / kAttendPiece + 2;
  }
  if (pieces < 1) pieces = 1;
  // Selected blocks: a row is one workgroup's, unless there are so few rows that those would read at the rate of a few compute units: then
  // about 512 workgroups, of a piece a wavefront at least.  (16 blocks of 64, bf16, us, whole -> in parts of 4 pieces: 1 token x 8 heads 14.4 -> 9.7,
  // 4 x 8 15.5 -> 12.2, 16 x 8 16.9 -> 21.8 (of 8: 18.9); 32 blocks of 128, 1 x 2 44 -> 11.3.)
  int64_t chunk = (pieces * rows + 511) / 512;
  if (chunk < 4) chunk = 4;
  if (s->topk == 0 || 2 * chunk > pieces || (rows > 64 && pieces <= 64)) chunk = pieces;
  // Every key: rows of up to 40 pieces, and many rows of a window, are a workgroup each; longer ones are cut evenly (see k_cache_attend_even).
  // (8 heads, bf16, us, whole -> even: 16 sequences of 1024 15.3 -> 19.1, one of 2048 22.0 -> 10.1, a window of 4096 x 64 sequences 170 -> 174; of 512 x 128, 4 heads,
  // e4m3, 13.2 -> 43.)  Not where there are too many rows for the launch that joins parts: whole ones fill the chip as well then.
  const int64_t joins = (int64_t)s->n_tokens * s->hq;
  const bool even = s->topk == 0 && pieces > 40 && s->nseq <= 4096 && !(window > 0 && rows >= 512) && launchable(joins, kJoinThreads);
  // Non-temporal loads where the keys and values are more than the 256 MB of the memory-side cache keep from one call to the next, and not for
  // new tokens of one sequence, which share blocks.  (16 blocks of 64, us, plain -> non-temporal: 256 tokens x 8 heads bf16, 1.05 GB, 183 -> 169; 32 x 8, 131 MB, 28.4
  // -> 25.8; 16 x 8, 66 MB, 16.9 -> 23.3; drafts of one to eight tokens, 524 MB read of half as much, 79 -> 94.)
  const int64_t piece_bytes = (int64_t)kAttendPiece * kD * (s->dtype == NSA_SEL_CACHE_E4M3 ? 2 : 4);
  const bool streaming = rows > (96ll << 20) / (pieces * piece_bytes) && s->n_tokens == s->nseq;
  c.chunk = (int)chunk;
  c.splits = (int)((pieces + chunk - 1) / chunk);
  c.even = even ? 512 : 0;
  if (c.even && rows > (((int64_t)1 << 31) - 1) / pieces * c.even) c.even = 0;  // a share is a 32-bit number
  c.streaming = streaming;
  c.slots = c.even ? 2 * (int64_t)c.even : c.splits > 1 ? rows * c.splits : 0;  // (parts of selected blocks: of fewer than 512 rows)
  const int64_t groups = c.group > 1 ? s->n_tokens / c.group + (int64_t)s->nseq : s->n_tokens;
  c.workgroups = c.even ? c.even : groups * s->hkv * c.splits;
  return c;
}
int check_cache_shape(const nsa_sel_cache_shape* s, bool attention) {
  const int rc = check_sizes(s, attention);
  return rc == NSA_SEL_OK && attention && !launchable(cut_of(s).workgroups, kAttendThreads) ? NSA_SEL_EUNSUPPORTED : rc;
}
struct CacheWs {
  size_t ml, rows, total;  // offsets; the sums come first
};
CacheWs cache_ws(const nsa_sel_cache_shape* s, const Cut& c) {
  CacheWs w = {0, 0, 0};
  if (c.slots == 0) return w;
  const size_t cols = (size_t)c.slots * c.group * (s->hq / s->hkv);
  w.ml = cols * kD * 4;
  w.rows = (w.ml + cols * 8 + 15) & ~(size_t)15;
  w.total = w.rows + (size_t)s->n_tokens * s->hkv * 16;
  return w;
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
                             interleaved != 0, Q_out, K_out, (hipStream_t)stream);
}

int nsa_sel_cache_workspace_bytes(const nsa_sel_cache_shape* shape, size_t* bytes) {
  int rc = check_cache_shape(shape, true);
  if (rc) return rc;
  if (bytes) *bytes = cache_ws(shape, cut_of(shape)).total;
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
  const CacheWs w = cache_ws(shape, c);
  if (w.total > 0 && !tensor(ws)) return NSA_SEL_EINVAL;
  if (ws_bytes < w.total) return NSA_SEL_EWORKSPACE;
  CacheAttend A;
  A.Q = Q;
  A.idx = idx;
  A.block = shape->topk > 0 ? shape->block : kBlock;
  A.topk = shape->topk;
  A.window = window_of(shape);
  A.scale = shape->scale > 0.f ? shape->scale : 0.08838834764831845f;  // 1/sqrt(128)
  A.gate = gate;
  A.o_acc = O_acc;
  A.O = O;
  A.LSE = LSE;
  A.group = c.group;
  A.splits = c.even ? 1 : c.splits;
  A.chunk = c.chunk;
  A.even = c.even;
  A.streaming = c.streaming;
  A.part = (float*)ws;
  A.part_ml = (float2*)((char*)ws + w.ml);
  A.rows = c.slots > 0 ? (int4*)((char*)ws + w.rows) : nullptr;
  A.cols = c.group * (shape->hq / shape->hkv);
  A.slots = (int)c.slots;
  A.slot_step = c.even ? 2 : 1;
  A.workgroups = (int)c.workgroups;
  const Cache C = make_cache(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  return launch_cache_attend(C, shape->dtype == NSA_SEL_CACHE_E4M3, A, (hipStream_t)stream) == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP;
}

}  // extern "C"
