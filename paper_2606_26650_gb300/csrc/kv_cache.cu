// kv_cache.cu — what a decode step does to the new tokens' queries, keys and values before attention:
// rotary positions given per token (catq_rope_at), and the append to the paged cache of 8-bit codes
// (catq_kv_append), which rotates the keys on the way and, in the same launch, the queries.
#include <cuda_fp16.h>

#include <algorithm>

#include "launch.h"
#include "ptx_sm100.cuh"
#include "rope.cuh"

namespace catq {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Eight consecutive elements (16-byte aligned) to and from fp32.
__device__ __forceinline__ void load8(const uint16_t* p, float* f) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float* f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store8(uint16_t* p, const float* f) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
__device__ __forceinline__ void store8(float* p, const float* f) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = static_cast<uint16_t>(pack2(v, 0.0f) & 0xffffu); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// ---------------------------------------------------------------- rotary positions
struct RopeAtArgs {
  const void* x;
  void* y;
  int64_t ldx, ldy;  // elements from a token's row to the next
  const int32_t* pos;
  int64_t T;
  int32_t nh, d;
  RotDev rot;
  bool inverse;
};

// One thread per (token, unit, run of `hpt` heads): its eight angles serve the run.
template <typename E>
__global__ void __launch_bounds__(kThreads) rope_at_vec_kernel(const RopeAtArgs a, int32_t hpt) {
  const int32_t units = a.d / 16, runs = (a.nh + hpt - 1) / hpt;
  const int64_t items = a.T * units * runs;
  const E* const x = static_cast<const E*>(a.x);
  E* const y = static_cast<E*>(a.y);
  for (int64_t e = blockIdx.x * (int64_t)kThreads + threadIdx.x; e < items; e += (int64_t)gridDim.x * kThreads) {
    const int32_t u = static_cast<int32_t>(e % units);
    const int64_t tr = e / units;
    const int32_t h0 = static_cast<int32_t>(tr % runs) * hpt, h1 = min(h0 + hpt, a.nh);
    const int64_t t = tr / runs;
    const RotUnit q = rot_unit(a.rot, u);
    if (!q.turned && a.x == a.y) continue;
    float c[8], s[8];
    if (q.turned) rot_angles(a.rot, u, a.pos[t], a.inverse, c, s);
    for (int32_t h = h0; h < h1; ++h) {
      float v[16];
      load8(x + t * a.ldx + h * a.d + q.a, v);
      load8(x + t * a.ldx + h * a.d + q.b, v + 8);
      if (q.turned) rot_apply(a.rot.interleaved != 0, c, s, v);
      store8(y + t * a.ldy + h * a.d + q.a, v);
      store8(y + t * a.ldy + h * a.d + q.b, v + 8);
    }
  }
}

// Any even rot and d, rows of the type's alignment: one thread per pair, or per element behind the rotated
// part.
template <typename E>
__global__ void __launch_bounds__(kThreads) rope_at_kernel(const RopeAtArgs a) {
  const int32_t half = a.rot.rot / 2, per = half + (a.d - a.rot.rot);
  const int64_t items = a.T * a.nh * per;
  const E* const x = static_cast<const E*>(a.x);
  E* const y = static_cast<E*>(a.y);
  for (int64_t e = blockIdx.x * (int64_t)kThreads + threadIdx.x; e < items; e += (int64_t)gridDim.x * kThreads) {
    const int32_t j = static_cast<int32_t>(e % per);
    const int64_t th = e / per, t = th / a.nh;
    const int64_t at = (th - t * a.nh) * a.d;
    const E* const xr = x + t * a.ldx + at;
    E* const yr = y + t * a.ldy + at;
    if (j >= half) {
      if (a.x != a.y) yr[half + j] = xr[half + j];
      continue;
    }
    float c, s;
    rot_cos_sin(a.pos[t], a.rot.turns[j], c, s);
    c *= a.rot.magnitude;
    s *= a.inverse ? -a.rot.magnitude : a.rot.magnitude;
    const int32_t i0 = a.rot.interleaved ? 2 * j : j, i1 = a.rot.interleaved ? 2 * j + 1 : j + half;
    const float p = load1(xr + i0), q = load1(xr + i1);
    store1(yr + i0, p * c - q * s);
    store1(yr + i1, p * s + q * c);
  }
}

// ---------------------------------------------------------------- append
// The scale of a page and head: the least power of two (2^-60 at least) that brings the largest magnitude,
// given as float bits, to 448 = 1.75 2^8 or below; 0 for 0, NaN for a magnitude that is not finite.
__device__ __forceinline__ float scale_of(uint32_t top) {
  if (top == 0u) return 0.0f;
  if (top >= 0x7f800000u) return __uint_as_float(0x7fffffffu);
  const int k = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float(static_cast<uint32_t>(max(k, -60) + 127) << 23);
}

__device__ __forceinline__ uint16_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// Eight values times `by` (a power of two: exact) as codes.
__device__ __forceinline__ uint2 codes8(const float* v, float by) {
  uint2 r;
  r.x = e4m3x2(v[0] * by, v[1] * by) | static_cast<uint32_t>(e4m3x2(v[2] * by, v[3] * by)) << 16;
  r.y = e4m3x2(v[4] * by, v[5] * by) | static_cast<uint32_t>(e4m3x2(v[6] * by, v[7] * by)) << 16;
  return r;
}

// Four codes times a power of two of at most 1, rounded to codes again.  Through fp16, where the products
// that round to anything but 0 (2^-10 and above) are exact; `by` is 2^-24 or more.
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, __half2 by) {
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint16_t two = static_cast<uint16_t>(codes >> (16 * i));
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
    __half2 p = __hmul2(*reinterpret_cast<const __half2*>(&h), by);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<const uint32_t*>(&p)));
    out |= static_cast<uint32_t>(r) << (16 * i);
  }
  return out;
}

__device__ __forceinline__ void latch_index_error(int32_t* status) { atomicCAS(status, 0, 10 /* CATQ_ERR_INDEX */); }

// Grid (sequence, key heads then value heads then query blocks, share of the sequence's pages): a CTA
// takes the tokens of one page at a time, twice: once for the largest magnitude, once for the codes.
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const KvAppendArgs a) {
  __shared__ uint32_t red[kThreads / 32];
  const int b = blockIdx.x;
  const int64_t r0 = a.row_start[b], r1 = a.row_start[b + 1];
  const int32_t len = a.seq_len[b];
  if (r0 < 0 || r1 < r0 || r1 > a.T || len < 0 || len > static_cast<int64_t>(a.cache.max_pages) * a.cache.page) {
    if (threadIdx.x == 0) latch_index_error(a.status);
    return;
  }
  const int32_t n = static_cast<int32_t>(r1 - r0), first = len - n;  // position of the sequence's row r0
  const int32_t d = a.cache.d, nkv = a.cache.nkv, page = a.cache.page, units = d / 16;
  if (static_cast<int>(blockIdx.y) >= 2 * nkv) {  // queries
    const int32_t per = a.nh * units;
    for (int64_t e = (blockIdx.z * static_cast<int64_t>(gridDim.y - 2 * nkv) + blockIdx.y - 2 * nkv) * kThreads +
                     threadIdx.x;
         e < static_cast<int64_t>(n) * per; e += static_cast<int64_t>(gridDim.z) * (gridDim.y - 2 * nkv) * kThreads) {
      const int32_t i = static_cast<int32_t>(e / per), hu = static_cast<int32_t>(e % per), u = hu % units;
      const RotUnit q = rot_unit(a.rot, u);
      const uint16_t* const x = a.q + (r0 + i) * a.ldq + (hu / units) * d;
      uint16_t* const y = a.q_out + (r0 + i) * a.ldqo + (hu / units) * d;
      float v[16], c[8], s[8];
      load8(x + q.a, v);
      load8(x + q.b, v + 8);
      if (q.turned) {
        rot_angles(a.rot, u, first + i, false, c, s);
        rot_apply(a.rot.interleaved != 0, c, s, v);
      }
      store8(y + q.a, v);
      store8(y + q.b, v + 8);
    }
    return;
  }
  const bool is_v = static_cast<int>(blockIdx.y) >= nkv;
  const int32_t h = blockIdx.y - (is_v ? nkv : 0);
  const uint16_t* const src = is_v ? a.v : a.k;
  const int64_t ld = is_v ? a.ldv : a.ldk;
  uint8_t* const codes = is_v ? a.cache.v_codes : a.cache.k_codes;
  float* const scales = is_v ? a.cache.v_scale : a.cache.k_scale;
  // the units of a row: values behind no rotation
  RotDev rot = a.rot;
  if (is_v) rot.rot = 0;
  const int32_t p0 = max(first, 0);
  for (int32_t pg = p0 / page + blockIdx.z; pg * page < len; pg += gridDim.z) {
    const int32_t lo = max(p0, pg * page), hi = min(len, (pg + 1) * page);
    const int32_t id = a.cache.table[static_cast<int64_t>(b) * a.cache.max_pages + pg];
    if (id < 0 || id >= a.cache.n_pages) {
      if (threadIdx.x == 0) latch_index_error(a.status);
      continue;
    }
    const int64_t block = static_cast<int64_t>(id) * nkv + h;
    uint8_t* const dst = codes + block * page * d;
    const int32_t kept = lo - pg * page, items = (hi - lo) * units;
    const float old = kept > 0 ? scales[block] : 0.0f;
    auto row = [&](int32_t e, float (&v)[16]) -> RotUnit {
      const int32_t i = e / units, u = e - i * units;
      const RotUnit q = rot_unit(rot, u);
      const uint16_t* const x = src + (r0 + lo - first + i) * ld + h * d;
      load8(x + q.a, v);
      load8(x + q.b, v + 8);
      if (q.turned) {
        float c[8], s[8];
        rot_angles(rot, u, lo + i, false, c, s);
        rot_apply(rot.interleaved != 0, c, s, v);
      }
      return q;
    };
    uint32_t top = 0;
    for (int32_t e = threadIdx.x; e < items; e += kThreads) {
      float v[16];
      row(e, v);
#pragma unroll
      for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    __syncthreads();  // red is free
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) top = max(top, red[w]);
    const float want = scale_of(top);
    const bool bad = !(want == want) || !(old == old);
    const float now = bad ? __uint_as_float(0x7fffffffu) : fmaxf(old, want);
    if (threadIdx.x == 0) scales[block] = now;
    if (!bad && kept > 0 && old > 0.0f && now > old) {
      const __half2 by = __float2half2_rn(fmaxf(old / now, 5.9604645e-8f));
      for (int32_t e = threadIdx.x; e < kept * d / 16; e += kThreads) {
        uint4 w = reinterpret_cast<const uint4*>(dst)[e];
        w.x = rescale4(w.x, by);
        w.y = rescale4(w.y, by);
        w.z = rescale4(w.z, by);
        w.w = rescale4(w.w, by);
        reinterpret_cast<uint4*>(dst)[e] = w;
      }
    }
    // a page that holds what is not finite has NaN as its scale, and finite codes
    const float by = bad ? 0.0f : (now > 0.0f ? 1.0f / now : 1.0f);
    for (int32_t e = threadIdx.x; e < items; e += kThreads) {
      float v[16];
      const RotUnit q = row(e, v);
      if (bad) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = 0.0f;
      }
      uint8_t* const at = dst + (kept + e / units) * d;
      *reinterpret_cast<uint2*>(at + q.a) = codes8(v, by);
      *reinterpret_cast<uint2*>(at + q.b) = codes8(v + 8, by);
    }
  }
}

int grid_for(int64_t n) {
  return static_cast<int>(std::min<int64_t>(std::max<int64_t>((n + kThreads - 1) / kThreads, 1), 152 * 16));
}

}  // namespace

cudaError_t launch_rope_at(const void* x, int64_t ldx, void* y, int64_t ldy, bool f32, const int32_t* pos, int64_t T,
                           int32_t nh, int32_t d, const RotDev& rot, bool inverse, cudaStream_t st) {
  const RopeAtArgs a{x, y, ldx, ldy, pos, T, nh, d, rot, inverse};
  const int64_t e = f32 ? 4 : 2;
  const bool vec = d % 16 == 0 && rot.rot % 16 == 0 && ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15u) == 0 &&
                   ldx * e % 16 == 0 && ldy * e % 16 == 0;
  if (vec) {
    int32_t hpt = 8;
    while (hpt > 1 && T * (d / 16) * ((nh + hpt - 1) / hpt) < 152 * 2048) hpt /= 2;
    const int grid = grid_for(T * (d / 16) * ((nh + hpt - 1) / hpt));
    if (f32)
      rope_at_vec_kernel<float><<<grid, kThreads, 0, st>>>(a, hpt);
    else
      rope_at_vec_kernel<uint16_t><<<grid, kThreads, 0, st>>>(a, hpt);
  } else {
    const int grid = grid_for(T * nh * (d - rot.rot / 2));
    if (f32)
      rope_at_kernel<float><<<grid, kThreads, 0, st>>>(a);
    else
      rope_at_kernel<uint16_t><<<grid, kThreads, 0, st>>>(a);
  }
  return cudaGetLastError();
}

cudaError_t launch_kv_append(KvAppendArgs a, cudaStream_t st) {
  WaitCtl wc;
  if (!launch_wait_ctl(&wc)) return cudaErrorInvalidDevice;
  a.status = wc.status_word;
  // shares of a sequence's pages: what an average sequence touches, and one (any number is right)
  const int64_t z = std::min<int64_t>(a.T / (static_cast<int64_t>(a.B) * a.cache.page) + 1, 1024);
  const int32_t qblocks = a.q ? std::max(1, a.nh * (a.cache.d / 16) / 64) : 0;
  kv_append_kernel<<<dim3(a.B, 2 * a.cache.nkv + qblocks, static_cast<unsigned>(z)), kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace catq
