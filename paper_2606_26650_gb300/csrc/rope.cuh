// rope.cuh — rotary positions at given tokens: the angle of a pair as a fraction of a turn in 64-bit
// fixed point, its sine and cosine, and the rotation of a unit of eight pairs, shared by the rotation
// itself and by the append to the key/value cache.
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

namespace catq {

// Device view of catq_rotation.
struct RotDev {
  const uint64_t* turns;  // [rot / 2]: turns a token, 2^64 one turn
  int32_t rot;            // rotated elements of a head
  int32_t interleaved;    // pairs (2i, 2i + 1), else (i, i + rot / 2)
  float magnitude;        // factor on the rotated elements
};

// cos and sin of pos * turn.  The product wraps modulo 2^64, which is modulo one turn, so that the angle
// of a far position is as exact as that of a near one (32-bit floats would lose 2^-24 of the whole angle:
// 0.008 rad at 131072).  Its upper 32 bits fall into the nearest quarter turn and a rest of at most an
// eighth, whose sine and cosine are their Taylor series up to x^9 and x^10 (remainders x^11 / 11! and
// x^12 / 12! at pi / 4: 1.8e-9 and 1.2e-10, under half a unit in the last place).
__device__ __forceinline__ void rot_cos_sin(int32_t pos, uint64_t turn, float& c, float& s) {
  const uint32_t frac = static_cast<uint32_t>((static_cast<uint64_t>(static_cast<int64_t>(pos)) * turn) >> 32);
  const uint32_t quarter = (frac + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(frac - (quarter << 30))) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float y = x * x;
  float sn = fmaf(y, 1.0f / 362880.0f, -1.0f / 5040.0f);
  sn = fmaf(y, sn, 1.0f / 120.0f);
  sn = fmaf(y, sn, -1.0f / 6.0f);
  sn = fmaf(x * y, sn, x);
  float cs = fmaf(y, -1.0f / 3628800.0f, 1.0f / 40320.0f);
  cs = fmaf(y, cs, -1.0f / 720.0f);
  cs = fmaf(y, cs, 1.0f / 24.0f);
  cs = fmaf(y, cs, -0.5f);
  cs = fmaf(y, cs, 1.0f);
  const float a = (quarter & 1u) ? sn : cs, b = (quarter & 1u) ? cs : sn;
  c = ((quarter + 1u) & 2u) ? -a : a;
  s = (quarter & 2u) ? -b : b;
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

// The unit's eight cosines and sines (times the magnitude; sines negated for the inverse).
__device__ __forceinline__ void rot_angles(const RotDev& r, int32_t u, int32_t pos, bool inverse, float (&c)[8],
                                           float (&s)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    rot_cos_sin(pos, __ldg(reinterpret_cast<const unsigned long long*>(r.turns) + 8 * u + j), c[j], s[j]);
    c[j] *= r.magnitude;
    s[j] *= inverse ? -r.magnitude : r.magnitude;
  }
}

// x[0..7] and x[8..15] (the unit's vectors a and b) rotated in place.
__device__ __forceinline__ void rot_apply(bool interleaved, const float (&c)[8], const float (&s)[8], float (&x)[16]) {
  if (interleaved) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = x[2 * j], q = x[2 * j + 1];
      x[2 * j] = p * c[j] - q * s[j];
      x[2 * j + 1] = p * s[j] + q * c[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = x[j], q = x[j + 8];
      x[j] = p * c[j] - q * s[j];
      x[j + 8] = p * s[j] + q * c[j];
    }
  }
}

}  // namespace catq
