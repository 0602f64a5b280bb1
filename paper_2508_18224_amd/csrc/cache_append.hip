// New keys and values into a paged cache, rotated by their places on the way, and the rotated queries beside them (nsa_sel_cache_append).
//
// Rotation by the place p: channels a, b of a pair i become  x_a cos(p f_i) - x_b sin(p f_i),  x_b cos(p f_i) + x_a sin(p f_i).  The angle
// is formed in 64 bits, in turns, less its nearest whole number, so that a place of 2^20 loses nothing; its sine and cosine are worked out in
// 64 bits too and rounded to 32, in which the rest is done.  Each product is rounded by itself, not fused into the sum, so that a
// value next to the border of two e4m3 values is stored as elementary 32-bit operations put it.
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

// The lane's 8 channels of a row after the rotation; cs: the row's table.  All 16 lanes of the row take part.  Channel e of the lane becomes
// x_e cos + o_e sin, where o is the other channel of its pair, with the sign that it has there.
__device__ __forceinline__ void rotate(const Rotation& R, u32x4 x, const float2* cs, float (&f)[8]) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63, c = lane & 15, half = R.rot >> 4;  // 8-channel pieces of half the pairs
  const bool low = c < half, turns = c < 2 * half;
  const int from = R.interleaved || !turns ? lane : low ? lane + half : lane - half;
  const uint32_t signs = R.interleaved ? 0x00008000u : low ? 0x80008000u : 0u;
  const int column = !turns ? 0 : R.interleaved || low ? c : c - half, columns = R.interleaved ? 2 * half : half;
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t o = lane_value(x[i], from);
    y[i] = (R.interleaved ? o >> 16 | o << 16 : o) ^ signs;
  }
  float o[8];
  unpack(x, f);
  unpack(y, o);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 t = cs[column + (R.interleaved ? e >> 1 : e) * columns];
    const float a = f[e] * t.x, b = o[e] * t.y, r = a + b;
    f[e] = turns ? r : f[e];
  }
}

// Where a row's table has pair p: the pairs that the lanes of a row read together lie side by side.
__device__ __forceinline__ int place_of_pair(const Rotation& R, int p) {
  return R.interleaved ? (p & 3) * (R.rot >> 3) + (p >> 2) : (p & 7) * (R.rot >> 4) + (p >> 3);
}

// ---- rows of tokens: queries, and the keys and values of a bf16 cache ------------------------------------------------------------------
// A workgroup takes the rows of kTokens consecutive tokens from t0, or with `parts` every parts-th step of them.  A thread requests
// kBatch rows before it waits for the angles.  Written with non-temporal stores: 32768 tokens, 32 + 2 x 8 heads, 805 MB 160 -> 152 us (5.3 TB/s; a copy
// of 1 GB runs at 5.1), 2048 tokens 11.8 -> 10.3; non-temporal loads gain only apart (168 -> 156 us with the pages' launch, 32768 tokens), and
// four tokens a workgroup only among pages in 8 bits (bf16: 2048 tokens 11.7 -> 14.8).
template <int kTokens>
struct RowsLds {
  float2 cs[kTokens * kMaxPairs];
  int place[kTokens], page[kTokens];  // place < 0: nothing to do
};
template <int kThreads, int kTokens, bool kStore, bool kApart = false>
__device__ __forceinline__ void token_rows(const Cache& C, const AppendArgs& A, int t0, int part, int parts, RowsLds<kTokens>& L) {
  constexpr int kRowsAtOnce = kThreads / 16, kBatch = 4;
  static_assert(kTokens <= kThreads / 64, "a wavefront a token");
  const int wave = threadIdx.x >> 6;
  if (wave < kTokens) {
    const int t = t0 + wave;
    const TokenPlace P = t < C.T ? token_place(C, t) : TokenPlace{-1, -1};
    const int place = P.s < 0 ? -1 : P.place;
    L.place[wave] = place;
    if constexpr (kStore) L.page[wave] = place < 0 ? -1 : page_of(C, P.s, place);
    for (int i = threadIdx.x & 63; i < A.R.rot >> 1; i += 64) {
      const double2 x = cos_sin(place, A.R.inv_freq[i]);
      L.cs[wave * kMaxPairs + place_of_pair(A.R, i)] = float2{(float)x.x, (float)x.y};
    }
  }
  const int sub = threadIdx.x & 15, nq = A.Q ? C.hq : 0, each = nq + (kStore ? 2 * C.hkv : 0), rows = min(kTokens, C.T - t0) * each;
  auto token_of = [&](int r) __attribute__((always_inline)) {  // r / each
    int k = 0;
#pragma unroll
    for (int i = 1; i < kTokens; ++i) k += r >= i * each ? 1 : 0;
    return k;
  };
  u32x4 x[kBatch];
  auto load = [&](int r) __attribute__((always_inline)) {
    const int k = token_of(r), h = r - k * each;
    const int64_t t = t0 + k;
    const bf16_t* src = h < nq ? A.Q + t * A.q_stride + h * kD
                        : h < nq + C.hkv ? A.K + t * A.k_stride + (h - nq) * kD : A.V + t * A.v_stride + (h - nq - C.hkv) * kD;
    return kApart ? load_streaming(src + 8 * sub) : *reinterpret_cast<const u32x4*>(src + 8 * sub);
  };
  const int step = parts * kRowsAtOnce;
  for (int at = part * kRowsAtOnce; at < rows; at += kBatch * step) {  // the same for the whole workgroup
    const int r = at + (threadIdx.x >> 4);
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (r + i * step < rows) x[i] = load(r + i * step);
    if (at == part * kRowsAtOnce) __syncthreads();
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (at + i * step >= rows) break;
      const int rn = r + i * step, rc = min(rn, rows - 1), k = token_of(rc), h = rc - k * each;
      const bool is_q = h < nq, is_k = !is_q && h < nq + C.hkv;
      const int64_t t = t0 + k;
      float f[8];
      rotate(A.R, x[i], L.cs + k * kMaxPairs, f);
      const u32x4 y = is_q || is_k ? pack(f) : x[i];
      const int place = L.place[k];
      if (rn >= rows || place < 0) continue;
      if (is_q) {
        store_streaming(A.Q_out + (t * C.hq + h) * kD + 8 * sub, y);
        continue;
      }
      if constexpr (kStore) {
        const int j = is_k ? h - nq : h - nq - C.hkv, page = L.page[k];
        if (is_k && A.K_out) store_streaming(A.K_out + (t * C.hkv + j) * kD + 8 * sub, y);
        if (page >= 0) {
          const int64_t row = (((int64_t)page * C.hkv + j) << C.page_log2) + (place & ((1 << C.page_log2) - 1));
          store_streaming(reinterpret_cast<bf16_t*>(is_k ? C.k : C.v) + row * kD + 8 * sub, y);
        }
      }
    }
  }
}

// kStore: with the keys and values of a bf16 cache.  Else the query rows apart, where the pages in 8 bits fill a launch of their own.
template <int kTokens, bool kStore>
__global__ void __launch_bounds__(kRowThreads) k_cache_append_rows(Cache C, AppendArgs A) {
  __shared__ RowsLds<kTokens> L;
  token_rows<kRowThreads, kTokens, kStore, !kStore>(C, A, (int)blockIdx.x * kTokens, (int)blockIdx.y, (int)gridDim.y, L);
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
__device__ __forceinline__ uint64_t to_e4m3(const float (&f)[8], float inverse) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float z = fminf(fmaxf(f[i] * inverse, -448.f), 448.f);
    y[i] = __builtin_fabsf(f[i]) < __builtin_inff() ? z : __builtin_nanf("");
  }
  const uint32_t lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false), true);
  return (uint64_t)hi << 32 | lo;
}
// Four e4m3 values times a power of two, rounded again.
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t x, float by) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * by, b[1] * by, __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * by, a[1] * by, 0, false), true);
}

// A workgroup takes the new tokens of one page for some KV heads, of K or of V, head by head: their largest magnitude, the page's scale, and, where
// the page held earlier tokens and the scale grew, those again.  Scales are powers of two so that this loses nothing but the last bits
// of values that become subnormal, less than 2^-17 of the page's largest.  Between the two steps kSteps rows of each 16 lanes stay in
// registers; a workgroup has as many threads as that takes for the new tokens of a page in the mean, and goes through the rows twice where a
// page gets more.
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
__device__ __forceinline__ void page_rows(const Cache& C, const AppendArgs& A, const PageUnit& U, int h0, int h1, float2* cs, float* most) {
  constexpr int kRowsAtOnce = kThreads / 16, kTileRows = kSteps * kRowsAtOnce;
  const int sub = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int64_t stride = kKey ? A.k_stride : A.v_stride;
  const bf16_t* src = (kKey ? A.K : A.V) + U.t0 * stride + 8 * sub;
  const int tiles = (U.rows + kTileRows - 1) / kTileRows;
  const int held = U.first & ((1 << C.page_log2) - 1);  // earlier tokens of the page
  auto rows_of = [&](int tile) { return min(kTileRows, U.rows - tile * kTileRows); };
  auto load = [&](int tile, int h, u32x4 (&x)[kSteps]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = i * kRowsAtOnce + rg;
      x[i] = u32x4{0u, 0u, 0u, 0u};
      if (r < rows_of(tile)) x[i] = *reinterpret_cast<const u32x4*>(src + (tile * kTileRows + r) * stride + h * kD);
    }
  };
  auto angles = [&](int tile) __attribute__((always_inline)) {
    if constexpr (kKey) {
#pragma unroll 1
      for (int k = threadIdx.x; k < rows_of(tile) * kMaxPairs; k += kThreads) {
        const int p = k & (kMaxPairs - 1), row = k / kMaxPairs;
        if (p < A.R.rot >> 1) {
          const double2 t = cos_sin(U.first + tile * kTileRows + row, A.R.inv_freq[p]);
          cs[row * kMaxPairs + place_of_pair(A.R, p)] = float2{(float)t.x, (float)t.y};
        }
      }
      __syncthreads();
    }
  };
  // the rows rotated; keys also leave as bf16 where that was asked for; their largest magnitude
  auto turn = [&](int tile, int h, bool write, const u32x4 (&x)[kSteps], float (&f)[kSteps][8]) __attribute__((always_inline)) {
    const int rows = rows_of(tile);
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i * kRowsAtOnce >= rows) break;  // the same for the whole workgroup
      __builtin_amdgcn_sched_barrier(0);   // one step's operands at a time
      const int r = i * kRowsAtOnce + rg;
      if constexpr (kKey) rotate(A.R, x[i], cs + min(r, rows - 1) * kMaxPairs, f[i]);
      else unpack(x[i], f[i]);
      if (r >= rows) continue;
      if (kKey && write && A.K_out)
        store_streaming(A.K_out + ((int64_t)(U.t0 + tile * kTileRows + r) * C.hkv + h) * kD + 8 * sub, pack(f[i]));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = __builtin_fabsf(f[i][e]);
        amax = a < __builtin_inff() ? fmaxf(amax, a) : amax;
      }
    }
    return amax;
  };
  // the page's scale for head h: its exponent; earlier tokens are rounded to it
  auto scale = [&](int h, float amax) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
    if constexpr (kThreads > 64) {
      if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = amax;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) amax = fmaxf(amax, most[w]);
    }
    float* at = (kKey ? C.ks : C.vs) + (int64_t)U.page * C.hkv + h;
    int e = scale_exponent(amax);
    if (held > 0) {
      const int e_old = min(max(exponent_of(*at), kScaleLeast), kScaleMost);
      if (e > e_old) {
        const float by = power_of_two(max(e_old - e, -126));
        u32x4* old = reinterpret_cast<u32x4*>((kKey ? C.k : C.v) + ((((int64_t)U.page * C.hkv + h) << C.page_log2) * kD));
        for (int i = threadIdx.x; i < held * (kD / 16); i += kThreads) {
          u32x4 x = old[i];
#pragma unroll
          for (int w = 0; w < 4; ++w) x[w] = rescale_e4m3(x[w], by);
          old[i] = x;
        }
      }
      e = max(e, e_old);
    }
    __syncthreads();  // every thread has read the old scale, and the largest magnitudes
    if (threadIdx.x == 0) *at = power_of_two(e);
    return e;
  };
  auto store = [&](int tile, int h, int e, const float (&f)[kSteps][8]) __attribute__((always_inline)) {
    char* to = (kKey ? C.k : C.v) + ((((int64_t)U.page * C.hkv + h) << C.page_log2) + held + tile * kTileRows) * kD + 8 * sub;
    const float inverse = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = i * kRowsAtOnce + rg;
      if (r < rows_of(tile)) __builtin_nontemporal_store(to_e4m3(f[i], inverse), reinterpret_cast<uint64_t*>(to + r * kD));
    }
  };
  // a head after the other; a page of one tile in one step, else its tiles twice: for the largest magnitude, and to be stored.  K_out is written
  // in the last round: it may be K itself.
  const int its = tiles == 1 || U.page < 0 ? tiles : 2 * tiles;
  u32x4 x[kSteps];
  float f[kSteps][8];
  load(0, h0, x);
#pragma unroll 1
  for (int h = h0; h < h1; ++h) {
    float amax = 0.f;
    int e = 0;
#pragma unroll 1
    for (int it = 0; it < its; ++it) {
      const int tile = it < tiles ? it : it - tiles;
      if (tiles > 1 || h == h0) {
        if (tiles > 1) __syncthreads();  // the last tile's angles have been read
        angles(tile);
      }
      amax = fmaxf(amax, turn(tile, h, it + tiles >= its, x, f));
      const bool last = it + 1 == its;
      if (!last || h + 1 < h1) load(last ? 0 : it + 1 < tiles ? it + 1 : it + 1 - tiles, last ? h + 1 : h, x);
      if (U.page < 0) continue;  // the same for the whole workgroup
      if (it == tiles - 1) e = scale(h, amax);
      if (tiles == 1 || it >= tiles) store(tile, h, e, f);
    }
  }
}

// Workgroups [0, n): pages of K, `heads` heads each; as many of V; then, with kTokens, the query rows of that many tokens each, in `parts` parts.
template <int kThreads, int kTokens>
__global__ void __launch_bounds__(kThreads, kThreads == 64 ? 3 : 4) k_cache_append_e4m3(Cache C, AppendArgs A, int units, int heads, int parts) {
  __shared__ float2 cs[kSteps * kThreads / 16 * kMaxPairs];
  __shared__ float most[kThreads / 64];
  const int of_head = (C.hkv + heads - 1) / heads, n = units * of_head;
  int b = (int)blockIdx.x;
  if constexpr (kTokens > 0) {
    static_assert(sizeof(RowsLds<kTokens>) <= sizeof(cs), "the query rows' angles must fit");
    if (b >= 2 * n) {
      b -= 2 * n;
      const int i = b / parts;
      token_rows<kThreads, kTokens, false>(C, A, i * kTokens, b - i * parts, parts, *reinterpret_cast<RowsLds<kTokens>*>(cs));
      return;
    }
  }
  const bool key = b < n;
  b -= key ? 0 : n;
  const int u = b / of_head, h0 = (b - u * of_head) * heads, h1 = min(h0 + heads, C.hkv);
  const PageUnit U = page_unit(C, u);
  if (U.rows <= 0 || U.t0 < 0) return;
  if (key) page_rows<kThreads, true>(C, A, U, h0, h1, cs, most);
  else page_rows<kThreads, false>(C, A, U, h0, h1, cs, most);
}

}  // namespace

int launch_cache_append(const Cache& C, bool e4m3, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
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
  const int each = (Q ? C.hq : 0) + (e4m3 ? 0 : 2 * C.hkv);
  auto status = [] { return hipGetLastError() == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP; };
  auto groups = [&](int tokens) { return ((int64_t)C.T + tokens - 1) / tokens; };
  auto rows = [&](auto kern, int tokens, int parts) {
    if (!launchable(groups(tokens), kRowThreads)) return NSA_SEL_EUNSUPPORTED;
    ProfScope ps(KID_CACHE_APPEND, st);
    hipLaunchKernelGGL(kern, dim3((unsigned)groups(tokens), (unsigned)parts), dim3(kRowThreads), 0, st, C, A);
    return status();
  };
  const bool many = C.T >= 4096;
  // a token's rows over as many as 512 workgroups
  auto parts_of = [&](int at_once) { return std::max(1, std::min((each + at_once - 1) / at_once, 512 / C.T)); };
  if (!e4m3) return rows(k_cache_append_rows<1, true>, 1, parts_of(kRowThreads / 16));
  // Pages in 8 bits.  Heads of a page share its angles where that leaves workgroups enough; and where the pages by themselves fill the chip
  // the query rows, which want more wavefronts than pages leave registers for, are a launch of their own.  (us, 32768 tokens, 32 + 8
  // heads: one launch, a head a workgroup 186 -> 167, in pages of 256 tokens 214 -> 185; 16000 tokens, 8 + 8 heads 69 -> 54; but 5900 tokens
  // in 7 sequences, 28 + 4 heads 32 -> 35, 4096 in one, 32 + 8, 30 -> 33.)
  const int64_t units = C.cu ? ((int64_t)C.T >> C.page_log2) + 2 * (int64_t)C.nseq : C.nseq;
  const int in_page = (int)std::min<int64_t>(1 << C.page_log2, C.T / std::max(C.nseq, 1));  // new tokens of a page, in the mean
  const int threads = many ? (in_page <= 64 ? 256 : in_page <= 128 ? 512 : 1024) : in_page <= 16 ? 64 : 256;
  const bool apart = many && Q && (units * C.hkv >= 2048 || threads == 1024);
  const int64_t share = units * C.hkv / (threads == 64 ? 1024 : 512);
  const int heads = (int)std::min<int64_t>(std::max<int64_t>(share, 1), C.hkv), parts = many ? 1 : parts_of(threads / 16);
  const int64_t row_groups = Q && !apart ? (many ? ((int64_t)C.T + 3) / 4 : (int64_t)C.T * parts) : 0;
  const int64_t grid = 2 * units * ((C.hkv + heads - 1) / heads) + row_groups;
  const auto kern = !many            ? (threads == 64 ? k_cache_append_e4m3<64, 1> : k_cache_append_e4m3<256, 1>)
                    : row_groups > 0 ? (threads == 256 ? k_cache_append_e4m3<256, 4> : k_cache_append_e4m3<512, 4>)
                                     : (threads == 256 ? k_cache_append_e4m3<256, 0> : threads == 512 ? k_cache_append_e4m3<512, 0> : k_cache_append_e4m3<1024, 0>);
  if (!launchable(grid, threads) || (apart && !launchable(groups(4), kRowThreads))) return NSA_SEL_EUNSUPPORTED;
  {
    ProfScope ps(KID_CACHE_APPEND, st);
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(threads), 0, st, C, A, (int)units, heads, parts);
  }
  const int rc = status();
  return rc == NSA_SEL_OK && apart ? rows(k_cache_append_rows<4, false>, 4, 1) : rc;
}

}  // namespace nsa
