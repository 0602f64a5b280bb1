// Keys and values of cached sequences as plain bf16 rows (nsa_sel_cache_read): a gather through the page table, times the page's scale in 8 bits, which bf16 holds exactly.
//
// Memory bound: every value is read once and written once.  A workgroup takes 16 consecutive rows of the result, all KV heads of K and of V: in a page the tokens of a
// head lie one after the other, in the result the heads of a token do, so that both sides move in runs of 256 bytes or more (128 in 8 bits).
// 131072 tokens of 8 heads: 206 us, 5.2 TB/s, which a large copy does not exceed; 4 to 32 tokens a workgroup and 2 to 8 rows at once are all within 2 %.
#include "cache_checks.h"

namespace nsa {
namespace {

constexpr int kReadThreads = 256, kReadTokens = 16, kReadBatch = 4;

struct ReadArgs {
  bf16_t *K, *V;
  int64_t k_stride, v_stride;  // between tokens
};

template <bool kE4m3>
__global__ void __launch_bounds__(kReadThreads) k_cache_read(Cache C, ReadArgs A) {
  __shared__ int2 where[kReadTokens];  // page and slot; a page of -1: no such place, zeros; of -2: no token
  const int t0 = (int)blockIdx.x * kReadTokens;
  if (threadIdx.x < 64) {
    const int t = t0 + (int)threadIdx.x;
    int s = t, place = -1;
    bool on = threadIdx.x < kReadTokens && t < C.T;
    if (C.cu == nullptr) {
      if (on) place = max(C.kv_len[t], kLeastLength) - 1;
    } else {
      // The first token's sequence, by all lanes; the others are in it too, or found by a search of their own.  Tokens of no sequence are before the first one's or
      // after the last one's.
      const int first = max(t0, C.cu[0]);
      s = find_sequence(C.nseq, first, [&](int i) { return (int64_t)C.cu[i]; });
      on = on && s >= 0 && t >= first && t < C.cu[C.nseq];
      if (on && t >= C.cu[s + 1]) {
        int lo = s + 1, hi = C.nseq;  // cu[lo] <= t < cu[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (C.cu[mid] <= t) lo = mid;
          else hi = mid;
        }
        s = lo;
      }
      if (on) place = max(C.kv_len[s], kLeastLength) - C.cu[s + 1] + t;
    }
    if (threadIdx.x < kReadTokens) where[threadIdx.x] = int2{on ? page_of(C, s, place) : -2, place & ((1 << C.page_log2) - 1)};
  }
  __syncthreads();
  const int sub = threadIdx.x & 15, i = threadIdx.x >> 4, rows = 2 * C.hkv;  // this thread's token; its rows: K's heads, then V's
  const int2 at = where[i];
  if (at.x == -2) return;
  const int64_t t = t0 + i;
  u32x4 x[kReadBatch];
  float scale[kReadBatch];
  for (int r0 = 0; r0 < rows; r0 += kReadBatch) {
#pragma unroll
    for (int b = 0; b < kReadBatch; ++b) {
      const int r = min(r0 + b, rows - 1), j = r < C.hkv ? r : r - C.hkv;
      const int64_t head = (int64_t)max(at.x, 0) * C.hkv + j, row = (head << C.page_log2) + at.y;
      const char* src = r < C.hkv ? C.k : C.v;
      x[b] = u32x4{0u, 0u, 0u, 0u};
      scale[b] = 1.f;
      if (at.x < 0) continue;
      if constexpr (kE4m3) {
        const uint2 y = *reinterpret_cast<const uint2*>(src + row * kD + 8 * sub);
        x[b][0] = y.x;
        x[b][1] = y.y;
        scale[b] = (r < C.hkv ? C.ks : C.vs)[head];
      } else {
        x[b] = *reinterpret_cast<const u32x4*>(src + row * (2 * kD) + 16 * sub);
      }
    }
#pragma unroll
    for (int b = 0; b < kReadBatch; ++b) {
      const int r = r0 + b;
      if (r >= rows) break;
      bf16_t* to = r < C.hkv ? A.K + t * A.k_stride + r * kD : A.V + t * A.v_stride + (r - C.hkv) * kD;
      if constexpr (kE4m3) x[b] = eight_bf16(x[b][0], x[b][1], scale[b]);
      *reinterpret_cast<u32x4*>(to + 8 * sub) = x[b];
    }
  }
}

}  // namespace
}  // namespace nsa

using namespace nsa;

extern "C" int nsa_sel_cache_read(const nsa_sel_cache_shape* shape, const int32_t* cu_seqlens, const int32_t* kv_len, const int32_t* table,
                                  const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, void* K,
                                  int64_t k_stride, void* V, int64_t v_stride, void* stream) {
  int rc = check_sizes(shape, false);
  if (rc) return rc;
  const int64_t groups = ((int64_t)shape->n_tokens + kReadTokens - 1) / kReadTokens;
  if (!launchable(groups, kReadThreads)) return NSA_SEL_EUNSUPPORTED;
  if (shape->n_tokens == 0) return NSA_SEL_OK;
  rc = check_cache_pointers(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  if (rc) return rc;
  const int64_t least = (int64_t)shape->hkv * kD;
  if (!tensor(K) || !tensor(V) || k_stride < least || v_stride < least || (k_stride & 7) || (v_stride & 7)) return NSA_SEL_EINVAL;
  const Cache C = make_cache(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  const ReadArgs A = {(bf16_t*)K, (bf16_t*)V, k_stride, v_stride};
  ProfScope ps(KID_CACHE_READ, (hipStream_t)stream);
  if (shape->dtype == NSA_SEL_CACHE_E4M3) hipLaunchKernelGGL(k_cache_read<true>, dim3((unsigned)groups), dim3(kReadThreads), 0, (hipStream_t)stream, C, A);
  else hipLaunchKernelGGL(k_cache_read<false>, dim3((unsigned)groups), dim3(kReadThreads), 0, (hipStream_t)stream, C, A);
  return hipGetLastError() == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP;
}
