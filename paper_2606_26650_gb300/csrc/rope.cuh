// rope.cuh — rotary positions at given tokens: the angle of a pair as a fraction of a turn in 64-bit
// fixed point, its sine and cosine, and the rotation of a unit of eight pairs, shared by the rotation
// itself and by the append to the key/value cache.
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

#include "catq_math.cuh"

namespace catq {

// Device view of catq_rotation.
struct RotDev {
  const uint64_t* turns;  // [rot / 2]: turns a token, 2^64 one turn
  int32_t rot;            // rotated elements of a head
  int32_t interleaved;    // pairs (2i, 2i + 1), else (i, i + rot / 2)
  float magnitude;        // factor on the rotated elements
};

// Pairs of fp32 values in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  unpack_f32x2(fma_f32x2(pack_f32x2(a.x, a.y), pack_f32x2(b.x, b.y), pack_f32x2(c.x, c.y)), d.x, d.y);
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  unpack_f32x2(mul_f32x2(pack_f32x2(a.x, a.y), pack_f32x2(b.x, b.y)), d.x, d.y);
  return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// cos and sin, times m, of pos * turn for two pairs.  The product wraps modulo 2^64, which is modulo one turn, so that
// the angle of a far position is as exact as that of a near one (32-bit floats would lose 2^-24 of the whole angle: 0.008
// rad at 131072).  Its upper 32 bits fall into the nearest half turn, which is a sign of both, and a rest of at most a
// quarter as x + e: x the upper 24 of its bits in radians, rounded to fp32, e the rounding and the lower 8 bits.  sin x
// and cos x are their Taylor series up to x^13 and x^14 (remainders x^15 / 15! and x^16 / 16! at pi / 2: 6.7e-10 and 6.6e-11),
// evaluated for the two pairs at once, sin(x + e) = sin x + e cos x, cos(x + e) = cos x - e sin x.  Over all rests either is
// off by 2^-22.84 at most, 2^-25.3 in the mean square, by the series' own roundings near pi / 2; without e by 2^-22.09 and
// 2^-24.85.  Quarter turns would save three terms and cost twice their instructions in exchanging sine and cosine.
__device__ __forceinline__ uint32_t turn_of(int32_t pos, uint64_t turn) {
  const uint32_t lo = static_cast<uint32_t>(turn), hi = static_cast<uint32_t>(turn >> 32);
  return __umulhi(static_cast<uint32_t>(pos), lo) + static_cast<uint32_t>(pos) * hi - (pos < 0 ? lo : 0u);
}
__device__ __forceinline__ void rot_cos_sin2(int32_t pos, uint64_t t0, uint64_t t1, float m, float2& c, float2& s) {
  const uint32_t f0 = turn_of(pos, t0), f1 = turn_of(pos, t1);
  const uint32_t h0 = (f0 + 0x40000000u) & 0x80000000u, h1 = (f1 + 0x40000000u) & 0x80000000u;
  constexpr float kUnit = 1.4629180792671596e-9f;                                      // 2 pi / 2^32 rounded to fp32,
  constexpr float kUnitLo = static_cast<float>(1.4629180792671596e-9 - static_cast<double>(kUnit));  // and what that leaves
  const float2 up = make_float2(static_cast<float>(static_cast<int32_t>((f0 ^ h0) & 0xffffff00u)),
                                static_cast<float>(static_cast<int32_t>((f1 ^ h1) & 0xffffff00u)));
  // the lower bits as 2^23 and more (the mantissa's last)
  const float2 low = make_float2(__uint_as_float(0x4b000000u | (f0 & 0xffu)), __uint_as_float(0x4b000000u | (f1 & 0xffu)));
  const float2 x = mul2(up, both(kUnit));
  const float2 off = fma2(up, both(kUnitLo), fma2(up, both(kUnit), make_float2(-x.x, -x.y)));
  const float2 e = fma2(fma2(low, both(kUnit), both(-8388608.0f * kUnit)), both(1.0f), off);
  const float2 y = mul2(x, x);
  float2 sn = fma2(y, both(1.0f / 6227020800.0f), both(-1.0f / 39916800.0f));
  sn = fma2(y, sn, both(1.0f / 362880.0f));
  sn = fma2(y, sn, both(-1.0f / 5040.0f));
  sn = fma2(y, sn, both(1.0f / 120.0f));
  sn = fma2(y, sn, both(-1.0f / 6.0f));
  sn = fma2(mul2(x, y), sn, x);
  float2 cs = fma2(y, both(-1.0f / 87178291200.0f), both(1.0f / 479001600.0f));
  cs = fma2(y, cs, both(-1.0f / 3628800.0f));
  cs = fma2(y, cs, both(1.0f / 40320.0f));
  cs = fma2(y, cs, both(-1.0f / 720.0f));
  cs = fma2(y, cs, both(1.0f / 24.0f));
  cs = fma2(y, cs, both(-0.5f));
  cs = fma2(y, cs, both(1.0f));
  const float2 sign = make_float2(__uint_as_float(__float_as_uint(m) ^ h0), __uint_as_float(__float_as_uint(m) ^ h1));
  c = mul2(fma2(make_float2(-e.x, -e.y), sn, cs), sign);
  s = mul2(fma2(e, cs, sn), sign);
}
__device__ __forceinline__ void rot_cos_sin(int32_t pos, uint64_t turn, float m, float& c, float& s) {
  float2 c2, s2;
  rot_cos_sin2(pos, turn, turn, m, c2, s2);
  c = c2.x;
  s = s2.x;
}

// A head of d = 16 n elements as units of 16: the two vectors of eight elements that a rotated unit pairs
// (rot a multiple of 16: 8u.. and rot / 2 + 8u.. in halves, 16u.. and 16u + 8.. interleaved), or 16
// consecutive elements behind the rotated part.
struct RotUnit {
  int32_t a, b;  // first element of either vector
  bool turned;
};
__device__ __forceinline__ RotUnit rot_unit(const RotDev& r, int32_t u) {
  RotUnit q;
  q.turned = 16 * u < r.rot;
  const bool halves = q.turned && !r.interleaved;
  q.a = halves ? 8 * u : 16 * u;
  q.b = halves ? r.rot / 2 + 8 * u : 16 * u + 8;
  return q;
}

// The unit's eight cosines and sines (times the magnitude; sines negated for the inverse) by pairs.
struct RotAngles {
  float2 c[4], s[4];
};
__device__ __forceinline__ void rot_angles(const RotDev& r, int32_t u, int32_t pos, bool inverse, RotAngles& a) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint64_t* const t = r.turns + 8 * u + 2 * j;
    rot_cos_sin2(pos, t[0], t[1], r.magnitude, a.c[j], a.s[j]);
    if (inverse) a.s[j] = make_float2(-a.s[j].x, -a.s[j].y);
  }
}

// (p, q) of two pairs rotated in place.
__device__ __forceinline__ void rot_pairs(float2 c, float2 s, float& p0, float& p1, float& q0, float& q1) {
  const float2 p = make_float2(p0, p1), q = make_float2(q0, q1);
  const float2 o = fma2(q, make_float2(-s.x, -s.y), mul2(p, c)), w = fma2(q, c, mul2(p, s));
  p0 = o.x; p1 = o.y;
  q0 = w.x; q1 = w.y;
}

// x[0..7] and x[8..15] (the unit's vectors a and b) rotated in place.
__device__ __forceinline__ void rot_apply(bool interleaved, const RotAngles& a, float (&x)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (interleaved)
      rot_pairs(a.c[j], a.s[j], x[4 * j], x[4 * j + 2], x[4 * j + 1], x[4 * j + 3]);
    else
      rot_pairs(a.c[j], a.s[j], x[2 * j], x[2 * j + 1], x[2 * j + 8], x[2 * j + 9]);
  }
}

// n / d for 0 <= n < 2^31 by one product: m = floor(2^(31 + l) / d) + 1 with l = ceil(log2 d), so that n m / 2^(31 + l)
// exceeds n / d by less than 1 / d.
struct Divisor {
  uint32_t m, shift;  // d == 1: m == 0
  __device__ __forceinline__ int32_t of(int32_t n) const {
    return m == 0u ? n : static_cast<int32_t>(__umulhi(static_cast<uint32_t>(n), m) >> shift);
  }
};
inline Divisor divisor(int32_t d) {
  if (d <= 1) return Divisor{0u, 0u};
  uint32_t l = 0;
  while ((int64_t(1) << l) < d) ++l;
  return Divisor{static_cast<uint32_t>((uint64_t(1) << (31 + l)) / static_cast<uint64_t>(d) + 1), l - 1};
}

}  // namespace catq
