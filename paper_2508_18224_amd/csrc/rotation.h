// Rotation by the place p, as the append to a cache (cache_append.hip) and the rotation by itself (rotary.hip) do it, bit for bit alike: channels a, b of
// a pair i become  x_a cos(p f_i) - x_b sin(p f_i),  x_b cos(p f_i) + x_a sin(p f_i), times a factor that cosine and sine have before they are rounded.  The angle is formed in 64 bits, in turns, less its nearest whole
// number, so that a place of 2^20 loses nothing; its sine and cosine are worked out in 64 bits too and rounded to 32, in which the rest is
// done.  Each product is rounded by itself, not fused into the sum, so that a value next to the border of two e4m3 values is stored
// as elementary 32-bit operations put it.
#pragma once
#include "common.h"

namespace nsa {

constexpr int kMaxPairs = kD / 2;

struct Rotation {
  const double* inv_freq;  // [rot / 2], radians per place
  int32_t rot;             // channels that turn, a multiple of 16
  int32_t interleaved;     // pairs (2 i, 2 i + 1); else (i, i + rot / 2)
  double factor;           // of the channels that turn
};

#if defined(__HIPCC__)
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
#endif

}  // namespace nsa
