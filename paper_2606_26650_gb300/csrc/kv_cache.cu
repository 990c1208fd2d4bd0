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

// Eight consecutive elements (16-byte aligned) from fp32.
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

// Eight elements as loaded, kept packed until they are needed.
template <typename E>
struct Eight;
template <>
struct Eight<uint16_t> {
  uint4 q;
  __device__ __forceinline__ void load(const uint16_t* p) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};

// Heads h0 .. h1 - 1 of one token, unit q, rotated by angles that are computed once: the first heads' loads go out
// before the angles, which cover their latency, and always kAhead heads' before any store.
template <typename E>
__device__ __forceinline__ void rotate_heads(const E* x, E* y, int32_t h0, int32_t h1, int32_t d, const RotDev& rot,
                                             int32_t u, const RotUnit& q, int32_t pos, bool inverse) {
  constexpr int kAhead = sizeof(E) == 2 ? 4 : 2;
  Eight<E> a[kAhead], b[kAhead];
  auto load = [&](int32_t h) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (h + k < h1) {
        a[k].load(x + (h + k) * d + q.a);
        b[k].load(x + (h + k) * d + q.b);
      }
  };
  load(h0);
  RotAngles ang;
  if (q.turned) rot_angles(rot, u, pos, inverse, ang);
  for (int32_t h = h0; h < h1; h += kAhead) {
    if (h > h0) load(h);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (h + k < h1) {
        float v[16];
        a[k].get(v);
        b[k].get(v + 8);
        if (q.turned) rot_apply(rot.interleaved != 0, ang, v);
        store8(y + (h + k) * d + q.a, v);
        store8(y + (h + k) * d + q.b, v + 8);
      }
  }
}

// Heads a thread takes at once: the longest run (fewest repeated angles) that still gives every SM a full set of
// threads.
int32_t heads_per_thread(int64_t tokens, int32_t nh, int32_t units) {
  int32_t hpt = 8;
  while (hpt > 1 && tokens * units * ((nh + hpt - 1) / hpt) < 152 * 2048) hpt /= 2;
  return hpt;
}

// One thread per (token, unit, run of `hpt` heads); `part` items a token (below 2^31), a CTA's tokens side by side.
template <typename E>
__global__ void __launch_bounds__(kThreads, 2) rope_at_vec_kernel(const RopeAtArgs a, int32_t hpt, Divisor by_units,
                                                                     Divisor by_part, int32_t part) {
  const int32_t units = a.d / 16;
  const E* const x = static_cast<const E*>(a.x);
  E* const y = static_cast<E*>(a.y);
  const int64_t items = a.T * part;
  for (int64_t e0 = blockIdx.x * (int64_t)kThreads; e0 < items; e0 += (int64_t)gridDim.x * kThreads) {
    const int64_t t0 = e0 / part;  // (the CTA's first token)
    const int32_t e = static_cast<int32_t>(e0 - t0 * part) + static_cast<int32_t>(threadIdx.x), over = by_part.of(e);
    const int64_t t = t0 + over;
    if (t >= a.T) continue;
    const int32_t ru = e - over * part, run = by_units.of(ru), u = ru - run * units;
    const RotUnit q = rot_unit(a.rot, u);
    if (!q.turned && a.x == a.y) continue;
    rotate_heads(x + t * a.ldx, y + t * a.ldy, run * hpt, min(run * hpt + hpt, a.nh), a.d, a.rot, u, q, a.pos[t],
                 a.inverse);
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
    rot_cos_sin(a.pos[t], a.rot.turns[j], a.rot.magnitude, c, s);
    if (a.inverse) s = -s;
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

// Maximum over an item's threads (whole warps).
template <int W>
__device__ __forceinline__ uint32_t item_max(uint32_t v, uint32_t* red) {
  v = __reduce_max_sync(0xffffffffu, v);
  if constexpr (W > 1) {
    __syncthreads();  // red is free
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) v = max(v, red[w]);
  }
  return v;
}

// An item is the new tokens of one page and head, keys or values: W warps hold its units (16 elements of a token), kHeld
// a thread, in registers between the search for the largest magnitude and the codes; an item of more units is read (and
// rotated) twice.  Grid (sequence, items then shares of the queries).  W = 1 serves calls of a token or a few a sequence:
// many items of little work, and no barrier; W = 8 whole pages.
// Bound by HBM where prompts are appended (an element read in 16 bits, written in 8, queries read and written), by
// latency where tokens are: row offsets, then page number, then scale.
template <int D, int W, int kHeld>
__global__ void __launch_bounds__(kThreads, 2) kv_append_kernel(const KvAppendArgs a, int32_t zkv, int32_t zq, int32_t hpt,
                                                                Divisor by_part, Divisor by_page) {
  constexpr int kItemThreads = 32 * W, d = D, units = D / 16;
  __shared__ uint32_t red[W];
  grid_launch_dependents();
  grid_dependency_wait();
  const int b = blockIdx.x;
  const int32_t tid = threadIdx.x % kItemThreads;
  const int64_t r0 = a.row_start[b], r1 = a.row_start[b + 1];
  const int32_t len = a.seq_len[b];
  const int32_t nkv = a.cache.nkv, page = a.cache.page;
  if (r0 < 0 || r1 < r0 || r1 > a.T || len < 0 || len > a.cache.max_pages * page) {
    if (threadIdx.x == 0) latch_index_error(a.status);
    return;
  }
  const int32_t n = static_cast<int32_t>(r1 - r0), first = len - n;  // position of the sequence's row r0
  const int32_t item_blocks = gridDim.y - zq;
  if (static_cast<int>(blockIdx.y) >= item_blocks) {  // queries
    const int32_t runs = (a.nh + hpt - 1) / hpt, per = runs * units;
    const int64_t items = static_cast<int64_t>(n) * per;
    for (int64_t e = static_cast<int64_t>(blockIdx.y - item_blocks) * kThreads + threadIdx.x; e < items;
         e += static_cast<int64_t>(zq) * kThreads) {
      const int32_t i = e >> 31 ? static_cast<int32_t>(e / per) : by_part.of(static_cast<int32_t>(e));
      const int32_t ru = static_cast<int32_t>(e - static_cast<int64_t>(i) * per);
      const int32_t run = ru / units, u = ru - run * units;
      const RotUnit q = rot_unit(a.rot, u);
      if (!q.turned && a.q == a.q_out) continue;
      rotate_heads(a.q + (r0 + i) * a.ldq, a.q_out + (r0 + i) * a.ldqo, run * hpt, min(run * hpt + hpt, a.nh), d, a.rot,
                   u, q, first + i, false);
    }
    return;
  }
  // item: share of the sequence's pages, head, keys or values
  const int32_t item = blockIdx.y * (kThreads / kItemThreads) + threadIdx.x / kItemThreads;
  const int32_t z = item / (2 * nkv), hv = item - z * 2 * nkv;
  if (z >= zkv) return;
  const bool is_v = hv >= nkv;
  const int32_t h = hv - (is_v ? nkv : 0);
  const int64_t ld = is_v ? a.ldv : a.ldk;
  const uint16_t* const src = (is_v ? a.v : a.k) + r0 * ld + h * d;
  uint8_t* const codes = is_v ? a.cache.v_codes : a.cache.k_codes;
  float* const scales = is_v ? a.cache.v_scale : a.cache.k_scale;
  RotDev rot = a.rot;
  if (is_v) rot.rot = 0;
  const int32_t p0 = max(first, 0);
  for (int32_t pg = by_page.of(p0) + z; pg * page < len; pg += zkv) {
    const int32_t lo = max(p0, pg * page), hi = min(len, (pg + 1) * page);
    const int32_t id = a.cache.table[static_cast<int64_t>(b) * a.cache.max_pages + pg];
    const int32_t kept = lo - pg * page, items = (hi - lo) * units;
    Eight<uint16_t> va[kHeld], vb[kHeld];
    auto fetch = [&](int32_t e, Eight<uint16_t>& x, Eight<uint16_t>& y) {
      const int32_t i = e / units;
      const RotUnit q = rot_unit(rot, e - i * units);
      const uint16_t* const row = src + (lo - first + i) * ld;
      x.load(row + q.a);
      y.load(row + q.b);
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (tid + k * kItemThreads < items) fetch(tid + k * kItemThreads, va[k], vb[k]);
    if (id < 0 || id >= a.cache.n_pages) {
      if (tid == 0) latch_index_error(a.status);
      continue;
    }
    const int64_t block = static_cast<int64_t>(id) * nkv + h;
    uint8_t* const dst = codes + block * page * d;
    const float old = kept > 0 ? scales[block] : 0.0f;
    // a unit's values
    auto turn = [&](int32_t e, const Eight<uint16_t>& x, const Eight<uint16_t>& y, float (&v)[16]) {
      x.get(v);
      y.get(v + 8);
      const int32_t i = e / units, u = e - i * units;
      if (16 * u < rot.rot) {
        RotAngles ang;
        rot_angles(rot, u, lo + i, false, ang);
        rot_apply(rot.interleaved != 0, ang, v);
      }
    };
    auto largest = [](const float (&v)[16], float top) {  // (NaN if any is)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(top) : "f"(top), "f"(fabsf(v[j])));
      return top;
    };
    float most = 0.0f;
    float v[kHeld][16];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (tid + k * kItemThreads < items) {
        turn(tid + k * kItemThreads, va[k], vb[k], v[k]);
        most = largest(v[k], most);
      }
    for (int32_t e = tid + kHeld * kItemThreads; e < items; e += kItemThreads) {
      Eight<uint16_t> x, y;
      float more[16];
      fetch(e, x, y);
      turn(e, x, y, more);
      most = largest(more, most);
    }
    const uint32_t top = item_max<W>(__float_as_uint(most) & 0x7fffffffu, red);
    const float want = scale_of(top);
    const bool bad = !(want == want) || !(old == old);
    const float now = bad ? __uint_as_float(0x7fffffffu) : fmaxf(old, want);
    if constexpr (W == 1) __syncwarp();  // (every thread has read the old scale: with more warps, item_max's barriers)
    if (tid == 0) scales[block] = now;
    if (!bad && old > 0.0f && now > old) {
      const __half2 by = __float2half2_rn(fmaxf(old / now, 5.9604645e-8f));
      for (int32_t e = tid; e < kept * d / 16; e += kItemThreads) {
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
    auto put = [&](int32_t e, float (&f)[16]) {
      const int32_t i = e / units;
      const RotUnit q = rot_unit(rot, e - i * units);
      uint8_t* const at = dst + (kept + i) * d;
      if (bad) {
#pragma unroll
        for (int j = 0; j < 16; ++j) f[j] = 0.0f;
      }
      *reinterpret_cast<uint2*>(at + q.a) = codes8(f, by);
      *reinterpret_cast<uint2*>(at + q.b) = codes8(f + 8, by);
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (tid + k * kItemThreads < items) put(tid + k * kItemThreads, v[k]);
    for (int32_t e = tid + kHeld * kItemThreads; e < items; e += kItemThreads) {
      Eight<uint16_t> x, y;
      float more[16];
      fetch(e, x, y);
      turn(e, x, y, more);
      put(e, more);
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
    const int32_t hpt = heads_per_thread(T, nh, d / 16);
    const int32_t part = (d / 16) * ((nh + hpt - 1) / hpt);
    const int grid = grid_for(T * part);
    if (f32)
      rope_at_vec_kernel<float><<<grid, kThreads, 0, st>>>(a, hpt, divisor(d / 16), divisor(part), part);
    else
      rope_at_vec_kernel<uint16_t><<<grid, kThreads, 0, st>>>(a, hpt, divisor(d / 16), divisor(part), part);
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
  // shares of a sequence's pages and queries: what an average sequence has of them (any number is right)
  const int32_t units = a.cache.d / 16;
  const int64_t each = (a.T + a.B - 1) / a.B;
  const int32_t zkv = static_cast<int32_t>(std::min<int64_t>((each + a.cache.page - 1) / a.cache.page, 32768 / (2 * a.cache.nkv)));
  const int32_t hpt = a.q ? heads_per_thread(a.T, a.nh, units) : 1, runs = a.q ? (a.nh + hpt - 1) / hpt : 0;
  const int32_t zq = a.q ? static_cast<int32_t>(std::min<int64_t>((each * runs * units + kThreads - 1) / kThreads, 4096)) : 0;
  // a warp for an item of up to 8 tokens, the CTA for longer ones (64 sequences, 32 / 8 heads of 128, one token each:
  // TODO us against TODO)
  const bool narrow = each <= 8;
  const int32_t items = 2 * a.cache.nkv * zkv, blocks = narrow ? (items + kThreads / 32 - 1) / (kThreads / 32) : items;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(a.B), static_cast<unsigned>(blocks + zq));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr{};  // the kernel waits by itself for the launch ahead
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const auto go = [&](auto kern) {
    return cudaLaunchKernelEx(&cfg, kern, a, zkv, zq, hpt, divisor(runs * units), divisor(a.cache.page));
  };
  const bool d128 = a.cache.d == 128;
  if (narrow) return d128 ? go(kv_append_kernel<128, 1, 2>) : go(kv_append_kernel<64, 1, 2>);
  if (a.cache.page * units <= 2 * kThreads) return d128 ? go(kv_append_kernel<128, 8, 2>) : go(kv_append_kernel<64, 8, 2>);
  return go(kv_append_kernel<128, 8, 4>);  // pages of 128 tokens of 128 elements
}

}  // namespace catq
