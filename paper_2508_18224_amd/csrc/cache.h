// What the kernels over a paged cache share (cache_append.hip, cache_attend.hip): its description, and the way from a workgroup's number
// to its sequence.  See nsa_sel_cache_append in include/nsa_sel.h for what the arrays mean.
#pragma once
#include "common.h"

namespace nsa {

constexpr int kAttendPiece = 32;  // keys of a step of the attention
constexpr int kScaleLeast = -100, kScaleMost = 119;  // exponents of a page's scale: both it and its reciprocal are normal numbers

struct Cache {
  char *k, *v;           // [n_pages, hkv, page, 128], 2 bytes a value or 1
  float *ks, *vs;        // [n_pages, hkv] (e4m3 only)
  const int32_t* table;  // [nseq, max_pages]
  const int32_t* kv_len; // [nseq]
  const int32_t* cu;     // [nseq + 1] or null: one new token a sequence
  int32_t T, nseq, hq, hkv, g, n_pages, max_pages, page_log2;
};

// HIP takes no launch of 2^32 work-items or more along a grid's dimension.
constexpr bool launchable(int64_t workgroups, int threads) { return workgroups <= (((int64_t)1 << 32) - 1) / threads; }
constexpr int kAttendThreads = 256, kJoinThreads = 256;

// Returns a status of the C ABI.
int launch_cache_append(const Cache& C, bool e4m3, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                               const void* V, int64_t v_stride, const double* inv_freq, int rot, bool interleaved, double factor, void* Q_out,
                               void* K_out, hipStream_t st);

// What the attention of a call reads besides the cache, and where its results go.
struct CacheAttend {
  const void* Q;
  const int32_t* idx;  // null: every key
  int32_t block, topk, window;
  float scale;
  const float* gate;   // null: plain
  const void* o_acc;
  void* O;
  float* LSE;
  int32_t group;       // new tokens of a sequence that a workgroup takes together
  int32_t splits;      // workgroups that may share the pieces of a row of selected blocks, `chunk` each
  int32_t chunk;
  int32_t even;        // else 0, or the number of workgroups that share all rows' pieces evenly
  bool streaming;      // keys and values come from memory and will not be read again soon
  // parts of rows, where a workgroup may have less than a whole one (else rows is null): slot i has `cols` columns, one for every token and head of a row
  float* part;         // [slots, cols, 128] sums
  float2* part_ml;     // [slots, cols] (maximum, sum)
  int4* rows;          // [T, hkv] first slot, second slot, number of parts, first token of the row
  int32_t slots, cols, slot_step;
  int32_t workgroups;
};
hipError_t launch_cache_attend(const Cache& C, bool e4m3, const CacheAttend& A, hipStream_t st);

#if defined(__HIPCC__)
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four e4m3 values times 2^e (the exponent of `scale`) as bf16.
__device__ __forceinline__ uint2 four_bf16(uint32_t x, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true);
  return {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}
__device__ __forceinline__ u32x4 eight_bf16(uint32_t lo, uint32_t hi, float scale) {
  const uint2 a = four_bf16(lo, scale), b = four_bf16(hi, scale);
  return u32x4{a.x, a.y, b.x, b.y};
}

// The s with base(s) <= u < base(s + 1) of a non-decreasing base: [0, n) is cut into 64 by the wavefront's lanes in every round.  -1 where
// u is outside.  All lanes of the wavefront take part and get the same result.
template <class Base>
__device__ __forceinline__ int find_sequence(int n, int64_t u, Base base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 0) {
    const int step = (len + 63) >> 6, at = lo + lane * step;
    const bool below = at < lo + len && base(at) <= u;
    const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));  // the first k probes are not above u
    if (k == 0) return -1;
    const int end = lo + len;
    lo += (k - 1) * step;
    len = min(step, end - lo);
    if (step == 1) break;
  }
  return u < base(lo + 1) ? lo : -1;
}

// Sequence of token t and its place there; s < 0 for tokens of no sequence (a padded batch's).
struct TokenPlace {
  int s, place;
};
__device__ __forceinline__ TokenPlace token_place(const Cache& C, int t) {
  TokenPlace r;
  if (C.cu == nullptr) {
    r.s = t;
    r.place = C.kv_len[t] - 1;
    return r;
  }
  r.s = find_sequence(C.nseq, t, [&](int s) { return (int64_t)C.cu[s]; });
  r.place = r.s < 0 ? -1 : C.kv_len[r.s] - C.cu[r.s + 1] + t;
  return r;
}

// Page of the place `at` of sequence s, or -1 where the table names none.
__device__ __forceinline__ int page_of(const Cache& C, int s, int at) {
  const int col = at >> C.page_log2;
  if (at < 0 || col >= C.max_pages) return -1;
  const int p = C.table[(int64_t)s * C.max_pages + col];
  return (uint32_t)p < (uint32_t)C.n_pages ? p : -1;
}
#endif

}  // namespace nsa
