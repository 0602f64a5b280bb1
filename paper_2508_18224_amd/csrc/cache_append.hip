// New keys and values into a paged cache, rotated by their places on the way, and the rotated queries beside them (nsa_sel_cache_append).
//
// Rotation by the place p: channels a, b of a pair i become  x_a cos(p f_i) - x_b sin(p f_i),  x_b cos(p f_i) + x_a sin(p f_i).  The angle
// is formed in 64 bits, in turns, less its nearest whole number, so that a place of 2^20 loses nothing.  What is stored as bf16 is then computed
// in 32 bits.  Keys for 8 bits are computed in 64 and rounded once: near the border of two e4m3 values an error of 2^-24 in the value is
// one of 2^-4 in what is stored.
//
// Memory bound: every value is read once and written once.  A row of 128 channels is 16 lanes with 16 bytes each; the partner of a
// lane's channels is in another lane of the row, or in the lane itself where pairs lie side by side.
#include <algorithm>

#include "cache.h"

namespace nsa {
namespace {

constexpr int kRowThreads = 256, kMaxPairs = kD / 2;

struct Rotation {
  const double* inv_freq;  // [rot / 2], radians per place
  int32_t rot;             // channels that turn, a multiple of 16
  int32_t interleaved;     // pairs (2 i, 2 i + 1); else (i, i + rot / 2)
};

struct AppendArgs {
  const bf16_t *Q, *K, *V;
  int64_t q_stride, k_stride, v_stride;  // between tokens
  bf16_t *Q_out, *K_out;
  Rotation R;
};

// (cos, sin) of the angle place * inv_freq, as exact as that product: a multiple of a quarter turn off, then Taylor's series on
// [-pi/4, pi/4], whose next terms are below 3e-14 and 1e-15.
__device__ __forceinline__ double2 cos_sin(int place, double inv_freq) {
  const double turns = (double)place * inv_freq * 0.15915494309189533577;
  const double r = turns - __builtin_rint(turns), quarters = __builtin_rint(4.0 * r);
  const double x = (r - 0.25 * quarters) * 6.283185307179586477, y = x * x;
  double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
  s = __builtin_fma(s, y, -1.0 / 39916800.0);
  c = __builtin_fma(c, y, 1.0 / 479001600.0);
  s = __builtin_fma(s, y, 1.0 / 362880.0);
  c = __builtin_fma(c, y, -1.0 / 3628800.0);
  s = __builtin_fma(s, y, -1.0 / 5040.0);
  c = __builtin_fma(c, y, 1.0 / 40320.0);
  s = __builtin_fma(s, y, 1.0 / 120.0);
  c = __builtin_fma(c, y, -1.0 / 720.0);
  s = __builtin_fma(s, y, -1.0 / 6.0);
  c = __builtin_fma(c, y, 1.0 / 24.0);
  s = __builtin_fma(s * y, x, x);
  c = __builtin_fma(__builtin_fma(c, y, -0.5), y, 1.0);
  const int q = (int)quarters;  // -2 .. 2
  const double co = (q & 1) ? s : c, si = (q & 1) ? c : s;
  return {((q + 1) & 2) ? -co : co, (q & 2) ? -si : si};
}

__device__ __forceinline__ void unpack(u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_lo(x[i]);
    f[2 * i + 1] = bf16_hi(x[i]);
  }
}
__device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  return r;
}

// 64-bit value as a float with the last bit set if that is not all of it: rounding that to fewer bits is rounding the value itself.
__device__ __forceinline__ float to_odd(double y) {
  const float f = (float)y;
  const double rest = y - (double)f;
  uint32_t u = __builtin_bit_cast(uint32_t, f);
  if (rest != 0.0 && f != 0.f && (u & 1) == 0) u += (rest > 0.0) == (f > 0.f) ? 1 : -1;
  return __builtin_bit_cast(float, u);
}
// u cos - v sin, in the precision of the angles
__device__ __forceinline__ float turned(float u, float v, float2 t) { return u * t.x - v * t.y; }
__device__ __forceinline__ float turned(float u, float v, double2 t) {
  return to_odd(__builtin_fma((double)u, t.x, -((double)v * t.y)));
}

// The lane's 8 channels of a row after the rotation; cs: the row's (cos, sin) by pair.  All 16 lanes of the row take part.
template <class Angle>
__device__ __forceinline__ void rotate(const Rotation& R, u32x4 x, const Angle* cs, float (&f)[8]) {
  const int lane = threadIdx.x & 63, c = lane & 15, half = R.rot >> 4;  // 8-channel pieces of half the pairs
  unpack(x, f);
  if (R.interleaved) {
    if (8 * c < R.rot) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Angle t = cs[4 * c + i];
        const float u = f[2 * i], v = f[2 * i + 1];
        f[2 * i] = turned(u, v, t);
        f[2 * i + 1] = turned(v, -u, t);
      }
    }
    return;
  }
  const bool low = c < half, high = !low && c < 2 * half;
  const int from = (lane & 48) + (low ? c + half : high ? c - half : c);
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = lane_value(x[i], from);
  if (low || high) {
    float o[8];
    unpack(y, o);
    const Angle* t = cs + 8 * (low ? c : c - half);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = turned(f[i], low ? o[i] : -o[i], t[i]);
  }
}

// (cos, sin) of `tokens` consecutive places for every pair, kMaxPairs apart, by the whole workgroup.
template <int kThreads, class Angle>
__device__ __forceinline__ void angles(const Rotation& R, int first, int tokens, Angle* cs) {
  const int pairs = R.rot >> 1;
  for (int i = threadIdx.x; i < tokens * kMaxPairs; i += kThreads) {
    const int p = i & (kMaxPairs - 1);
    if (p < pairs) {
      const double2 t = cos_sin(first + i / kMaxPairs, R.inv_freq[p]);
      cs[i].x = t.x;
      cs[i].y = t.y;
    }
  }
}

// ---- rows of tokens: queries, and the keys and values of a bf16 cache ------------------------------------------------------------------
// A workgroup takes the rows of one token, or with blockIdx.y the part of them that is its own.
template <int kThreads, bool kStore>
__device__ __forceinline__ void token_rows(const Cache& C, const AppendArgs& A, int t, int part, int parts, float2* cs) {
  const TokenPlace P = token_place(C, t);
  if (P.s < 0 || P.place < 0) return;  // the same for the whole workgroup
  constexpr int kRowsAtOnce = kThreads / 16;
  angles<kThreads>(A.R, P.place, 1, cs);
  const int page = kStore ? page_of(C, P.s, P.place) : -1;
  __syncthreads();
  const int sub = threadIdx.x & 15, nq = A.Q ? C.hq : 0, rows = nq + (kStore ? 2 * C.hkv : 0);
  for (int r0 = part * kRowsAtOnce; r0 < rows; r0 += parts * kRowsAtOnce) {
    const int r = r0 + (threadIdx.x >> 4), rc = min(r, rows - 1);
    const bool is_q = rc < nq, is_k = !is_q && rc < nq + C.hkv;
    const int h = is_q ? rc : is_k ? rc - nq : rc - nq - C.hkv;
    const bf16_t* src = is_q ? A.Q + (int64_t)t * A.q_stride : is_k ? A.K + (int64_t)t * A.k_stride : A.V + (int64_t)t * A.v_stride;
    u32x4 x = *reinterpret_cast<const u32x4*>(src + h * kD + 8 * sub);
    float f[8];
    rotate(A.R, x, cs, f);
    if (is_q || is_k) x = pack(f);
    if (r >= rows) continue;
    if (is_q) {
      *reinterpret_cast<u32x4*>(A.Q_out + ((int64_t)t * C.hq + h) * kD + 8 * sub) = x;
      continue;
    }
    if constexpr (kStore) {
      if (is_k && A.K_out) *reinterpret_cast<u32x4*>(A.K_out + ((int64_t)t * C.hkv + h) * kD + 8 * sub) = x;
      if (page >= 0) {
        const int64_t row = (((int64_t)page * C.hkv + h) << C.page_log2) + (P.place & ((1 << C.page_log2) - 1));
        *reinterpret_cast<u32x4*>((is_k ? C.k : C.v) + row * (2 * kD) + 16 * sub) = x;
      }
    }
  }
}

__global__ void __launch_bounds__(kRowThreads) k_cache_append_rows(Cache C, AppendArgs A) {
  __shared__ float2 cs[kMaxPairs];
  token_rows<kRowThreads, true>(C, A, (int)blockIdx.x, (int)blockIdx.y, (int)gridDim.y, cs);
}

// ---- pages in 8 bits -----------------------------------------------------------------------------------------------------------
// Exponent of the least scale 2^e with amax <= 448 * 2^e.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __builtin_bit_cast(uint32_t, amax);
  const int e = (int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);  // 448 = 1.75 * 2^8
  return min(max(e, kScaleLeast), kScaleMost);
}
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
__device__ __forceinline__ int exponent_of(float s) { return (int)((__builtin_bit_cast(uint32_t, s) >> 23) & 255) - 127; }

// 8 values in the page's scale as e4m3, rounded to nearest.  What is beyond 448 after scaling (values of 2^127 and more) saturates;
// infinities and NaN become NaN.
__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8], float inverse) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float z = fminf(fmaxf(f[i] * inverse, -448.f), 448.f);
    y[i] = __builtin_fabsf(f[i]) < __builtin_inff() ? z : __builtin_nanf("");
  }
  uint2 r;
  r.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
  r.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false), true);
  return r;
}
// Four e4m3 values times a power of two, rounded again.
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t x, float by) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * by, b[1] * by, __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * by, a[1] * by, 0, false), true);
}

// A workgroup takes the new tokens of one page for one KV head, of K or of V: their largest magnitude, the page's scale, and, where the
// page held earlier tokens and the scale grew, those again.  Scales are powers of two so that this loses nothing but the last bits of
// values that become subnormal, less than 2^-17 of the page's largest.  Between the two steps kSteps rows of each 16 lanes stay in
// registers; a workgroup has as many threads as that takes for a whole page where pages fill up in the mean, else 256, and goes through the
// rows twice where a page gets more.
constexpr int kSteps = 4;
struct PageUnit {
  int s, t0, first, rows, page;  // sequence, first new token and its place, new tokens in the page
};
__device__ __forceinline__ PageUnit page_unit(const Cache& C, int u) {
  PageUnit U;
  U.rows = 0;
  int c0, n, i;
  if (C.cu == nullptr) {
    U.s = c0 = u;
    n = 1;
    i = 0;
  } else {
    // a sequence's units start at floor(cu / size) + 2 s: room for every page that it can touch, without a scan over the batch
    auto base = [&](int s) { return (int64_t)(C.cu[s] >> C.page_log2) + 2 * s; };
    U.s = find_sequence(C.nseq, u, base);
    if (U.s < 0) return U;
    c0 = C.cu[U.s];
    n = C.cu[U.s + 1] - c0;
    i = u - (int)base(U.s);
  }
  const int start = C.kv_len[U.s] - n;  // place of the sequence's first new token
  const int lo = max(start, 0), page0 = (lo >> C.page_log2) + i;
  U.first = i == 0 ? lo : page0 << C.page_log2;
  const int end = min(start + n, (page0 + 1) << C.page_log2);
  U.t0 = c0 + (U.first - start);
  U.rows = min(end - U.first, C.T - U.t0);
  U.page = U.rows > 0 && U.t0 >= 0 ? page_of(C, U.s, U.first) : -1;
  return U;
}

template <int kThreads, bool kKey>
__device__ __forceinline__ void page_rows(const Cache& C, const AppendArgs& A, const PageUnit& U, int h, double2* cs) {
  constexpr int kRowsAtOnce = kThreads / 16, kTileRows = kSteps * kRowsAtOnce;
  const int sub = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const bf16_t* src = kKey ? A.K : A.V;
  const int64_t stride = kKey ? A.k_stride : A.v_stride;
  const int tiles = (U.rows + kTileRows - 1) / kTileRows;
  float f[kSteps][8];
  // the rows of tile `tile`, rotated; keys also leave as bf16 where that was asked for
  auto load = [&](int tile, bool write) __attribute__((always_inline)) {
    const int r0 = tile * kTileRows, rows = min(kTileRows, U.rows - r0);
    u32x4 x[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = i * kRowsAtOnce + rg;
      x[i] = u32x4{0u, 0u, 0u, 0u};
      if (r < rows) x[i] = *reinterpret_cast<const u32x4*>(src + (int64_t)(U.t0 + r0 + r) * stride + h * kD + 8 * sub);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i * kRowsAtOnce >= rows) break;  // the same for the whole workgroup
      if constexpr (kKey) {
        const int r = i * kRowsAtOnce + rg, n = min(kRowsAtOnce, rows - i * kRowsAtOnce);
        if (i > 0 || tile > 0 || !write) __syncthreads();  // what was there has been read
        angles<kThreads>(A.R, U.first + r0 + i * kRowsAtOnce, n, cs);
        __syncthreads();
        rotate(A.R, x[i], cs + min(rg, n - 1) * kMaxPairs, f[i]);
        if (write && A.K_out && r < rows)
          *reinterpret_cast<u32x4*>(A.K_out + ((int64_t)(U.t0 + r0 + r) * C.hkv + h) * kD + 8 * sub) = pack(f[i]);
      } else {
        unpack(x[i], f[i]);
      }
    }
  };
  float amax = 0.f;
  for (int tile = 0; tile < tiles; ++tile) {
    load(tile, true);
    const int rows = min(kTileRows, U.rows - tile * kTileRows);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i * kRowsAtOnce >= rows) break;
      if (i * kRowsAtOnce + rg < rows) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float a = __builtin_fabsf(f[i][e]);
          amax = a < __builtin_inff() ? fmaxf(amax, a) : amax;
        }
      }
    }
  }
  if (U.page < 0) return;  // the same for the whole workgroup
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
  float* most = reinterpret_cast<float*>(cs);
  __syncthreads();  // the angles have been read
  if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) amax = fmaxf(amax, most[w]);
  float* scale = (kKey ? C.ks : C.vs) + (int64_t)U.page * C.hkv + h;
  const int held = U.first & ((1 << C.page_log2) - 1);  // earlier tokens of the page
  int e = scale_exponent(amax), e_old = e;
  if (held > 0) {
    e_old = min(max(exponent_of(*scale), kScaleLeast), kScaleMost);
    e = max(e, e_old);
  }
  char* pages = (kKey ? C.k : C.v) + ((((int64_t)U.page * C.hkv + h) << C.page_log2) * kD);
  if (e > e_old) {
    const float by = power_of_two(max(e_old - e, -126));
    for (int i = threadIdx.x; i < held * (kD / 16); i += kThreads) {
      u32x4* at = reinterpret_cast<u32x4*>(pages) + i;
      u32x4 x = *at;
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] = rescale_e4m3(x[w], by);
      *at = x;
    }
  }
  const float inverse = power_of_two(-e);
  for (int tile = 0; tile < tiles; ++tile) {
    if (tiles > 1) load(tile, false);
    const int r0 = tile * kTileRows, rows = min(kTileRows, U.rows - r0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = i * kRowsAtOnce + rg;
      if (r < rows) *reinterpret_cast<uint2*>(pages + (held + r0 + r) * kD + 8 * sub) = to_e4m3(f[i], inverse);
    }
  }
  __syncthreads();  // every thread has read the old scale
  if (threadIdx.x == 0) *scale = power_of_two(e);
}

// Workgroups [0, units * hkv): pages of K; as many of V; then the query rows, a token each.
template <int kThreads>
__global__ void __launch_bounds__(kThreads) k_cache_append_e4m3(Cache C, AppendArgs A, int units) {
  __shared__ double2 cs[kThreads / 16 * kMaxPairs];
  const int n = units * C.hkv;
  int b = (int)blockIdx.x;
  if (b >= 2 * n) {
    token_rows<kThreads, false>(C, A, b - 2 * n, 0, 1, reinterpret_cast<float2*>(cs));
    return;
  }
  const bool key = b < n;
  b -= key ? 0 : n;
  const int u = b / C.hkv, h = b - u * C.hkv;
  const PageUnit U = page_unit(C, u);
  if (U.rows <= 0 || U.t0 < 0) return;
  if (key) page_rows<kThreads, true>(C, A, U, h, cs);
  else page_rows<kThreads, false>(C, A, U, h, cs);
}

}  // namespace

hipError_t launch_cache_append(const Cache& C, bool e4m3, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                               const void* V, int64_t v_stride, const double* inv_freq, int rot, bool interleaved, void* Q_out,
                               void* K_out, hipStream_t st) {
  AppendArgs A;
  A.Q = (const bf16_t*)Q;
  A.K = (const bf16_t*)K;
  A.V = (const bf16_t*)V;
  A.q_stride = q_stride;
  A.k_stride = k_stride;
  A.v_stride = v_stride;
  A.Q_out = (bf16_t*)Q_out;
  A.K_out = (bf16_t*)K_out;
  A.R.inv_freq = inv_freq;
  A.R.rot = rot;
  A.R.interleaved = interleaved ? 1 : 0;
  ProfScope ps(KID_CACHE_APPEND, st);
  if (!e4m3) {
    hipLaunchKernelGGL(k_cache_append_rows, dim3((unsigned)C.T, 1), dim3(kRowThreads), 0, st, C, A);
  } else {
    const int64_t units = C.cu ? ((int64_t)C.T >> C.page_log2) + 2 * (int64_t)C.nseq : C.nseq;
    const int64_t grid = 2 * units * C.hkv + (Q ? C.T : 0);
    const int rows = (int)std::min<int64_t>(1 << C.page_log2, C.T / std::max(C.nseq, 1));  // new tokens of a page, in the mean
    const int threads = rows <= 64 ? 256 : rows <= 128 ? 512 : 1024;
    const auto kern = threads == 256 ? k_cache_append_e4m3<256> : threads == 512 ? k_cache_append_e4m3<512> : k_cache_append_e4m3<1024>;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(threads), 0, st, C, A, (int)units);
  }
  return hipGetLastError();
}

}  // namespace nsa
