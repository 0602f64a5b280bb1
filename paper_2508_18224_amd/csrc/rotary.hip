// Queries and keys of a packed batch turned by their places (nsa_sel_rotary; the rotation is that of rotation.h), and turned back: the gradient of a rotation is the
// rotation by the negative angle, with the same factor, so the backward pass is the same kernel.
//
// Memory bound: every value is read once and written once, 20 KB a token of 32 + 8 heads, while the angles of a token are worked out once for all its
// rows.  A row of 128 channels is 16 lanes with 16 bytes each.  A workgroup takes one token, or as many as give its threads two rows each; a thread has two
// rows on their way while the angles are made.  Small workgroups come and go more evenly: 65536 tokens of 40 heads, forward and back, 470 us (5.7 TB/s) with 128 threads of two rows,
// 501 with 256, 520 with 256 of four, 643 with 512, 484 with 64.  (Stores that leave no copy in the caches: 553; 72 instead of 87 for 15000 tokens, which the
// caches hold, but who reads the result next wants it there.)
#include "cache.h"
#include "rotation.h"

namespace nsa {
namespace {

constexpr int kThreads = 128, kAtOnce = kThreads / 16, kBatch = 2, kMostTokens = 8;

struct RotaryArgs {
  const bf16_t *Q, *K;
  bf16_t *Q_out, *K_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;  // between tokens
  const int32_t *cu, *positions;
  int32_t T, nseq, hq, each, tokens;  // each: rows of a token; tokens: of a workgroup
  uint32_t each_magic;                // see div_g
  bool inverse;
  Rotation R;
};

// Place of token t, the same in all lanes of the wavefront; false for tokens of no sequence.
__device__ __forceinline__ bool place_of(const RotaryArgs& A, int t, int& place) {
  if (A.positions) {
    place = A.positions[t];
    return true;
  }
  place = t;
  if (A.cu == nullptr) return true;
  int s = 0;
  if (A.nseq > 1) {
    s = find_sequence(A.nseq, t, [&](int i) { return (int64_t)A.cu[i]; });
  } else if (t < A.cu[0] || t >= A.cu[1]) {
    s = -1;
  }
  if (s >= 0) place = t - A.cu[s];
  return s >= 0;
}

__global__ void __launch_bounds__(kThreads) k_rotary(RotaryArgs A) {
  __shared__ float2 cs[kMostTokens * kMaxPairs];
  __shared__ int turns[kMostTokens];
  const int t0 = (int)blockIdx.x * A.tokens, n = min(A.tokens, A.T - t0), rows = n * A.each;
  const int wave = threadIdx.x >> 6, sub = threadIdx.x & 15;
  u32x4 x[kBatch];
  auto load = [&](int r) __attribute__((always_inline)) {
    const int k = div_g(r, A.each, A.each_magic), h = r - k * A.each;
    const int64_t t = t0 + k;
    const bf16_t* src = h < A.hq ? A.Q + t * A.q_stride + h * kD : A.K + t * A.k_stride + (h - A.hq) * kD;
    return *reinterpret_cast<const u32x4*>(src + 8 * sub);
  };
  for (int at = 0; at < rows; at += kBatch * kAtOnce) {  // the same for the whole workgroup
    const int r = at + (threadIdx.x >> 4);
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (r + i * kAtOnce < rows) x[i] = load(r + i * kAtOnce);
    if (at == 0) {
      for (int k = wave; k < n; k += kThreads / 64) {
        int place;
        const bool on = place_of(A, t0 + k, place);
        if ((threadIdx.x & 63) == 0) turns[k] = on;
        for (int i = threadIdx.x & 63; i < A.R.rot >> 1; i += 64) {
          const double2 c = cos_sin(place, A.R.inv_freq[i]);
          cs[k * kMaxPairs + place_of_pair(A.R, i)] = float2{(float)(c.x * A.R.factor), (float)((A.inverse ? -c.y : c.y) * A.R.factor)};
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (at + i * kAtOnce >= rows) break;
      const int rn = r + i * kAtOnce, rc = min(rn, rows - 1), k = div_g(rc, A.each, A.each_magic), h = rc - k * A.each;
      const int64_t t = t0 + k;
      float f[8];
      rotate(A.R, x[i], cs + k * kMaxPairs, f);
      const u32x4 y = turns[k] ? pack(f) : x[i];
      if (rn >= rows) continue;
      *reinterpret_cast<u32x4*>((h < A.hq ? A.Q_out + t * A.q_out_stride + h * kD : A.K_out + t * A.k_out_stride + (h - A.hq) * kD) + 8 * sub) = y;
    }
  }
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace
}  // namespace nsa

using namespace nsa;

extern "C" int nsa_sel_rotary(const nsa_sel_rotary_shape* shape, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                              const int32_t* cu_seqlens, const int32_t* positions, const double* inv_freq, void* Q_out,
                              int64_t q_out_stride, void* K_out, int64_t k_out_stride, void* stream) {
  const nsa_sel_rotary_shape* s = shape;
  if (!s || s->n_tokens < 0 || s->nseq < 0 || s->hq < 1 || s->hkv < 0) return NSA_SEL_EINVAL;
  if (s->rot < 0 || s->rot > kD || (s->rot & 15) != 0 || !(s->factor < __builtin_inf())) return NSA_SEL_EINVAL;  // (a NaN too)
  if (s->d != kD || (int64_t)s->hq + s->hkv > 65536) return NSA_SEL_EUNSUPPORTED;
  if (s->n_tokens == 0) return NSA_SEL_OK;
  if (s->nseq < 1 && !positions) return NSA_SEL_EINVAL;
  if (!cu_seqlens && !positions && s->nseq != 1) return NSA_SEL_EINVAL;
  if (!Q || !Q_out || !aligned(Q, 16) || !aligned(Q_out, 16) || !aligned(cu_seqlens, 4) || !aligned(positions, 4)) return NSA_SEL_EINVAL;
  if (s->hkv > 0 ? !K || !K_out || !aligned(K, 16) || !aligned(K_out, 16) : K || K_out) return NSA_SEL_EINVAL;
  if (s->rot > 0 && (!inv_freq || !aligned(inv_freq, 8))) return NSA_SEL_EINVAL;
  const int64_t q = (int64_t)s->hq * kD, k = (int64_t)s->hkv * kD;
  auto apart = [](int64_t stride, int64_t least) { return stride >= least && (stride & 7) == 0; };
  if (!apart(q_stride, q) || !apart(q_out_stride, q) || (Q == Q_out && q_stride != q_out_stride)) return NSA_SEL_EINVAL;
  if (K && (!apart(k_stride, k) || !apart(k_out_stride, k) || (K == K_out && k_stride != k_out_stride))) return NSA_SEL_EINVAL;
  RotaryArgs A;
  A.Q = (const bf16_t*)Q;
  A.K = (const bf16_t*)K;
  A.Q_out = (bf16_t*)Q_out;
  A.K_out = (bf16_t*)K_out;
  A.q_stride = q_stride;
  A.k_stride = k_stride;
  A.q_out_stride = q_out_stride;
  A.k_out_stride = k_out_stride;
  A.cu = positions ? nullptr : cu_seqlens;
  A.positions = positions;
  A.T = s->n_tokens;
  A.nseq = s->nseq;
  A.hq = s->hq;
  A.each = s->hq + s->hkv;
  A.each_magic = A.each == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / (uint32_t)A.each + 1);
  const int want = kAtOnce * kBatch / A.each;
  A.tokens = want < 1 ? 1 : want > kMostTokens ? kMostTokens : want;
  A.inverse = s->inverse != 0;
  A.R.inv_freq = inv_freq;
  A.R.rot = s->rot;
  A.R.interleaved = s->interleaved != 0;
  A.R.factor = s->factor > 0.0 ? s->factor : 1.0;
  const int64_t groups = ((int64_t)A.T + A.tokens - 1) / A.tokens;
  if (!launchable(groups, kThreads)) return NSA_SEL_EUNSUPPORTED;
  ProfScope ps(KID_ROTARY, (hipStream_t)stream);
  hipLaunchKernelGGL(k_rotary, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, A);
  return hipGetLastError() == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP;
}
