// kv_cache.cu — what a decode step does to the new tokens' queries, keys and values before attention:
// rotary positions given per token (catq_rope_at), and the append to the paged cache of 8-bit codes
// (catq_kv_append), which rotates the keys on the way and, in the same launch, the queries.
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

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
// before the angles, which cover their latency, and always kAhead heads' before any store.  (A head's offset has 64 bits: a
// row may have 2^32 elements.)
template <typename E>
__device__ __forceinline__ void rotate_heads(const E* x, E* y, int32_t h0, int32_t h1, int32_t d, const RotDev& rot,
                                             int32_t u, const RotUnit& q, int32_t pos, bool inverse) {
  constexpr int kAhead = sizeof(E) == 2 ? 4 : 2;
  Eight<E> a[kAhead], b[kAhead];
  auto load = [&](int32_t h) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (h + k < h1) {
        a[k].load(x + static_cast<int64_t>(h + k) * d + q.a);
        b[k].load(x + static_cast<int64_t>(h + k) * d + q.b);
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
        store8(y + static_cast<int64_t>(h + k) * d + q.a, v);
        store8(y + static_cast<int64_t>(h + k) * d + q.b, v + 8);
      }
  }
}

// Heads a thread takes at once: the longest run (fewest repeated angles) that still gives every SM six warps.  us by runs
// of 1 / 2 / 4 / 8: 32 heads of 128 in bf16, 64 tokens 2.7 / 2.8 / 3.2 / 4.2, 256 3.6 / 3.0 / 3.3 / 4.3, 512 5.2 / 4.1 / 3.4 /
// 4.4, 2048 13.8 / 9.4 / 7.1 / 6.2, 8192 47.6 / 31.9 / 26.0 / 24.5; 16 heads of 64, 1024 tokens 3.4 / 2.9 / 3.4 / 4.5; an append
// with queries (32 / 8 heads of 128), 512 tokens 8.7 / 7.1 / 6.7 / 6.7, 4 x 2048 69.8 / 50.6 / 43.9 / 40.3.  fp32, of which only two
// heads are loaded ahead, in runs of 4 at most: 4096 tokens 29.5 / 24.6 / 24.1 / 22.9, 8192 52.8 / 43.7 / 42.6 / 44.3.
int32_t heads_per_thread(int64_t tokens, int32_t nh, int32_t units, int32_t most) {
  int32_t hpt = most;
  while (hpt > 1 && tokens * units * ((nh + hpt - 1) / hpt) < 152 * 192) hpt /= 2;
  return hpt;
}

// One thread per (token, unit, run of `hpt` heads); `part` items a token (below 2^31), a CTA's tokens side by side.
// Bound by HBM: 8192 tokens of 32 heads of 128 in bf16 take 23.6 us for 134 MB, 5.7 TB/s (a copy of the same bytes 21.6), 4999
// of 40 heads in fp32 39 us, 5.2 TB/s.  Two CTAs an SM with four heads' loads ahead (by runs of four heads 25 us): three with four
// or two ahead (80 registers) 31 and 26 us, four with two 27, two with eight 30.
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
// part (the 8192 tokens 103 us; 64 tokens 2.8 like the vector kernel).
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

// The work of one append is three lines of items, each in the order of the sequences: pages that get few tokens (a team of
// one or two warps takes one head's keys or values of such a page), pages that get more (a CTA), and the queries in chunks
// of kThreads units of 16 elements.  Lengths are read on the device and every CTA adds them up, so that a batch of single
// tokens with a long prompt among them is shared out like any other: 128 single tokens and a prompt of 512 (32 / 8 heads of
// 128, pages of 64) take 10 us, where a grid over sequences and shares of the mean one's pages took 97 to 135; single
// tokens alone pay 0.7 us for it (64 sequences: 4.5).
// Few tokens are 64 units a warp of the team, so that its lanes hold two.
struct KvSpan {
  int64_t r0;
  int32_t n, first, len;         // new rows, position of the first, cached tokens with them
  int32_t pg, pages;             // first page that gets tokens, their number
  int32_t head_small, tail_small;  // whether the first and (another) last page are a warp's
  int32_t chunks;                // of the queries
};

template <int D, int kTeam>
struct KvAppendWork {
  static constexpr int kUnits = D / 16, kSmall = 32 * kTeam * 2 / kUnits;  // tokens of a team's item at most
  const KvAppendArgs& a;
  Divisor by_page;
  int32_t per;  // units of a token's queries, in runs of heads; 0: no queries
  __device__ __forceinline__ KvSpan span(int32_t b, bool latch) const {
    KvSpan s;
    s.r0 = a.row_start[b];
    const int64_t r1 = a.row_start[b + 1];
    s.len = a.seq_len[b];
    s.pages = 0;
    s.chunks = 0;
    s.n = 0;
    s.head_small = s.tail_small = 0;
    const int32_t page = a.cache.page;
    if (s.r0 < 0 || r1 < s.r0 || r1 > a.T || s.len < 0 || s.len > a.cache.max_pages * page) {
      if (latch) latch_index_error(a.status);
      return s;
    }
    s.n = static_cast<int32_t>(r1 - s.r0);
    s.first = s.len - s.n;
    s.chunks = static_cast<int32_t>((static_cast<int64_t>(s.n) * per + kThreads - 1) / kThreads);
    const int32_t p0 = max(s.first, 0);
    if (p0 >= s.len) return s;
    s.pg = by_page.of(p0);
    const int32_t last = by_page.of(s.len - 1);
    s.pages = last - s.pg + 1;
    s.head_small = min(s.len, (s.pg + 1) * page) - p0 <= kSmall;
    s.tail_small = s.pages > 1 && s.len - last * page <= kSmall;
    return s;
  }
  // Items of line l (0: warps' pages, 1: CTAs' pages, 2: chunks of the queries) of a sequence.
  __device__ __forceinline__ int32_t count(const KvSpan& s, int l) const {
    if (l == 2) return s.chunks;
    const int32_t small = a.cache.page <= kSmall ? s.pages : s.head_small + s.tail_small;
    return l == 0 ? small : s.pages - small;
  }
  // Page k of the sequence's share of line l.
  __device__ __forceinline__ int32_t page_of(const KvSpan& s, int l, int32_t k) const {
    if (a.cache.page <= kSmall) return s.pg + k;
    if (l == 1) return s.pg + s.head_small + k;
    return k == 0 && s.head_small ? s.pg : s.pg + s.pages - 1;
  }
};

// Maximum over an item's threads: W warps, which meet at barrier `bar`.
template <int W>
__device__ __forceinline__ uint32_t item_max(uint32_t v, uint32_t* red, int bar) {
  v = __reduce_max_sync(0xffffffffu, v);
  const int warp = threadIdx.x >> 5, team = warp / W * W;
  asm volatile("barrier.cta.sync %0, %1;" ::"r"(bar), "n"(32 * W) : "memory");  // red is free
  if ((threadIdx.x & 31) == 0) red[warp] = v;
  asm volatile("barrier.cta.sync %0, %1;" ::"r"(bar), "n"(32 * W) : "memory");
#pragma unroll
  for (int w = 0; w < W; ++w) v = max(v, red[team + w]);
  return v;
}

// One item: the new tokens of a page and one head, keys or values.
struct KvItem {
  const uint16_t* src;  // first token
  int32_t lo, tokens;   // position of it, their number
  int32_t kept;         // tokens that the page has already
  int32_t id, h;        // page number, head
  bool is_v;
};

__device__ __forceinline__ KvItem item_of(const KvAppendArgs& a, const KvSpan& s, int32_t b, int32_t pg, int32_t hv) {
  KvItem t;
  t.is_v = hv >= a.cache.nkv;
  t.h = hv - (t.is_v ? a.cache.nkv : 0);
  t.lo = max(max(s.first, 0), pg * a.cache.page);
  t.tokens = min(s.len, (pg + 1) * a.cache.page) - t.lo;
  t.kept = t.lo - pg * a.cache.page;
  t.id = a.cache.table[static_cast<int64_t>(b) * a.cache.max_pages + pg];
  const int64_t row = s.r0 + (t.lo - s.first);
  t.src = (t.is_v ? a.v + row * a.ldv : a.k + row * a.ldk) + t.h * a.cache.d;
  return t;
}

// The vectors of an item's unit e.
template <int D>
__device__ __forceinline__ RotUnit item_unit(const KvAppendArgs& a, const KvItem& t, int32_t e, const uint16_t*& row) {
  constexpr int units = D / 16;
  RotDev rot = a.rot;
  if (t.is_v) rot.rot = 0;
  const int32_t i = e / units;
  row = t.src + i * (t.is_v ? a.ldv : a.ldk);
  return rot_unit(rot, e - i * units);
}

// An item by W warps (thread tid of them), kHeld units a thread, which stay in registers between the search for the largest
// magnitude and the codes.  load(k, e, x, y) gives unit e, the thread's k-th, turn(k, u, position, angles) its angles; then()
// is called when all have been taken.
template <int D, int W, int kHeld, class Load, class Turn, class Then>
__device__ __forceinline__ void append_item(const KvAppendArgs& a, const KvItem& t, int32_t tid, uint32_t* red, int bar, Load load, Turn turn,
                                            Then then) {
  constexpr int kItemThreads = 32 * W, d = D, units = D / 16;
  const int32_t nkv = a.cache.nkv, page = a.cache.page, items = t.tokens * units;
  uint8_t* const codes = t.is_v ? a.cache.v_codes : a.cache.k_codes;
  float* const scales = t.is_v ? a.cache.v_scale : a.cache.k_scale;
  const bool known = t.id >= 0 && t.id < a.cache.n_pages;
  const int64_t block = known ? static_cast<int64_t>(t.id) * nkv + t.h : 0;
  uint8_t* const dst = codes + block * page * d;
  const float old = known && t.kept > 0 ? scales[block] : 0.0f;
  RotDev rot = a.rot;
  if (t.is_v) rot.rot = 0;
  Eight<uint16_t> va[kHeld], vb[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int32_t e = tid + k * kItemThreads;
    if (e < items) load(k, e, va[k], vb[k]);
  }
  float most = 0.0f;
  float v[kHeld][16];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int32_t e = tid + k * kItemThreads, i = e / units, u = e - i * units;
    if (e < items) {
      va[k].get(v[k]);
      vb[k].get(v[k] + 8);
      if (16 * u < rot.rot) {
        RotAngles ang;
        turn(k, u, t.lo + i, ang);
        rot_apply(rot.interleaved != 0, ang, v[k]);
      }
#pragma unroll
      for (int j = 0; j < 16; ++j)  // (NaN if any is)
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(most) : "f"(most), "f"(fabsf(v[k][j])));
    }
  }
  then(most);
  if (!known) {
    if (tid == 0) latch_index_error(a.status);
    return;
  }
  const uint32_t top = item_max<W>(__float_as_uint(most) & 0x7fffffffu, red, bar);  // (everyone has read the old scale)
  const float want = scale_of(top);
  const bool bad = !(want == want) || !(old == old);
  const float now = bad ? __uint_as_float(0x7fffffffu) : fmaxf(old, want);
  if (tid == 0) scales[block] = now;
  if (!bad && old > 0.0f && now > old) {
    const __half2 by = __float2half2_rn(fmaxf(old / now, 5.9604645e-8f));
    for (int32_t e = tid; e < t.kept * d / 16; e += kItemThreads) {
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
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int32_t e = tid + k * kItemThreads, i = e / units;
    if (e < items) {
      const RotUnit q = rot_unit(rot, e - i * units);
      uint8_t* const at = dst + (t.kept + i) * d;
      if (bad) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[k][j] = 0.0f;
      }
      *reinterpret_cast<uint2*>(at + q.a) = codes8(v[k], by);
      *reinterpret_cast<uint2*>(at + q.b) = codes8(v[k] + 8, by);
    }
  }
}

__device__ __forceinline__ void copy16(void* smem, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem)), "l"(global) : "memory");
}

// CTAs below ctas_kv take keys and values, a run of whole pages and heads each, the next one's elements on their way to
// shared memory meanwhile (each thread copies what it will read itself), and the angles of a page's tokens kept there
// from its first head on (four us less for four prompts of 2048); the others chunks of the queries.
// Four prompts of 2048 (32 / 8 heads of 128) move 185 MB in 40 us, 4.6 TB/s, bound by the latency of an item (elements,
// maximum over the CTA, codes) and the arithmetic beside it; single tokens by a chain of loads: row offsets, page
// number, scale.  kHeld kThreads units: a page and head at most.
template <int D, int kTeam, int kHeld>
__global__ void __launch_bounds__(kThreads, 2) kv_append_kernel(const KvAppendArgs a, uint32_t ctas_kv, int32_t hpt,
                                                                Divisor by_part, Divisor by_page, Divisor by_heads) {
  constexpr int kWarps = kThreads / 32, kTeams = kWarps / kTeam, units = D / 16;
  extern __shared__ uint4 staged[];  // [kHeld][2][kThreads], then the angles [kHeld][4][kThreads]
  float4* const angles = reinterpret_cast<float4*>(staged + 2 * kHeld * kThreads);
  __shared__ uint32_t red[kWarps];
  __shared__ int32_t upto[3][kThreads];  // items of each line in the stretches of sequences up to thread t's
  __shared__ int32_t sums[3][kWarps];
  grid_launch_dependents();
  grid_dependency_wait();
  const int32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t runs = a.q ? (a.nh + hpt - 1) / hpt : 0, heads = 2 * a.cache.nkv;
  const KvAppendWork<D, kTeam> work{a, by_page, runs * units};
  const int32_t stretch = (a.B + kThreads - 1) / kThreads;  // sequences a thread
  {
    int32_t mine[3] = {0, 0, 0};
    const int32_t b0 = min(tid * stretch, a.B), b1 = min(b0 + stretch, a.B);
#pragma unroll 1
    for (int32_t b = b0; b < b1; ++b) {
      const KvSpan s = work.span(b, blockIdx.x == 0);
#pragma unroll
      for (int l = 0; l < 3; ++l) mine[l] += work.count(s, l);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
      for (int l = 0; l < 3; ++l) {
        const int32_t v = __shfl_up_sync(0xffffffffu, mine[l], o);
        if (lane >= o) mine[l] += v;
      }
    }
#pragma unroll
    for (int l = 0; l < 3; ++l)
      if (lane == 31) sums[l][warp] = mine[l];
    __syncthreads();
#pragma unroll
    for (int l = 0; l < 3; ++l) {
#pragma unroll
      for (int w = 0; w < kWarps - 1; ++w) mine[l] += w < warp ? sums[l][w] : 0;
      upto[l][tid] = mine[l];
    }
    __syncthreads();
  }
  // The sequence of item k of line l, which becomes the place in the sequence's share.  By whole warps.
  auto locate = [&](int l, int32_t& k, KvSpan& s) {
    const int32_t eighth = min(__popc(__ballot_sync(0xffffffffu, upto[l][8 * lane + 7] <= k)), 31);
    const int32_t t = 8 * eighth + __popc(__ballot_sync(0xffffffffu, lane < 8 && upto[l][8 * eighth + (lane & 7)] <= k));
    if (t > 0) k -= upto[l][min(t, kThreads) - 1];
    int32_t b = min(t * stretch, a.B - 1);
    s = work.span(b, false);
#pragma unroll 1
    for (int32_t n; k >= (n = work.count(s, l)) && b + 1 < a.B; k -= n) s = work.span(++b, false);
    return b;
  };
  auto page_at = [&](int64_t e) {
    return e < 0x7fffffff ? by_heads.of(static_cast<int32_t>(e)) : static_cast<int32_t>(e / heads);
  };
  auto item_at = [&](int l, int64_t e) {
    int32_t k = page_at(e);
    const int32_t hv = static_cast<int32_t>(e - static_cast<int64_t>(k) * heads);
    KvSpan s;
    const int32_t b = locate(l, k, s);
    KvItem t{a.k, 0, 0, 0, -1, 0, false};
    if (k >= 0 && k < work.count(s, l)) t = item_of(a, s, b, work.page_of(s, l, k), hv);  // (else lengths changed meanwhile)
    return t;
  };
  if (blockIdx.x < ctas_kv) {
    const int64_t small = static_cast<int64_t>(upto[0][kThreads - 1]) * heads, big = static_cast<int64_t>(upto[1][kThreads - 1]) * heads;
#pragma unroll 1
    for (int64_t e = blockIdx.x * static_cast<int64_t>(kTeams) + warp / kTeam; e < small; e += ctas_kv * static_cast<int64_t>(kTeams)) {
      const KvItem t = item_at(0, e);
      append_item<D, kTeam, 2>(a, t, tid % (32 * kTeam), red, 1 + warp / kTeam, [&](int, int32_t at, Eight<uint16_t>& x, Eight<uint16_t>& y) {
        const uint16_t* row;
        const RotUnit q = item_unit<D>(a, t, at, row);
        x.load(row + q.a);
        y.load(row + q.b);
      }, [&](int, int32_t u, int32_t pos, RotAngles& g) { rot_angles(a.rot, u, pos, false, g); }, [](float) {});
    }
    auto stage = [&](const KvItem& t) {
      int32_t mine = tid;
      asm volatile("" : "+r"(mine));  // (nothing that follows from the thread alone is kept over the loop)
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const int32_t at = mine + k * kThreads;
        if (at < t.tokens * units) {
          const uint16_t* row;
          const RotUnit q = item_unit<D>(a, t, at, row);
          copy16(&staged[2 * k * kThreads + mine], row + q.a);
          copy16(&staged[(2 * k + 1) * kThreads + mine], row + q.b);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // (from the other end, where the line before left CTAs free)
    const int64_t run = (big + ctas_kv - 1) / ctas_kv, end = min((ctas_kv - blockIdx.x) * run, big);
    int64_t e = (ctas_kv - 1 - blockIdx.x) * run;
    if (e >= end) return;
    KvItem t = item_at(1, e);
    stage(t);
    int32_t have = -1;  // page (of the line) whose angles are kept
    int32_t page = page_at(e);
#pragma unroll 1
    for (bool more = true; more;) {
      ++e;
      more = e < end;
      const KvItem next = item_at(1, more ? e : e - 1);
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      int32_t mine = tid;
      asm volatile("" : "+r"(mine));
      append_item<D, kWarps, kHeld>(a, t, mine, red, 0, [&](int k, int32_t, Eight<uint16_t>& x, Eight<uint16_t>& y) {
        x.q = staged[(2 * k) * kThreads + mine];
        y.q = staged[(2 * k + 1) * kThreads + mine];
      }, [&](int k, int32_t u, int32_t pos, RotAngles& g) {
        float4* const kept = angles + k * 4 * kThreads + mine;
        if (have != page) {
          rot_angles(a.rot, u, pos, false, g);
#pragma unroll
          for (int j = 0; j < 4; ++j) kept[j * kThreads] = make_float4(g.c[j].x, g.c[j].y, g.s[j].x, g.s[j].y);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float4 w = kept[j * kThreads];
            g.c[j] = make_float2(w.x, w.y);
            g.s[j] = make_float2(w.z, w.w);
          }
        }
      }, [&](float most) {
        asm volatile("" ::"f"(most) : "memory");  // what was staged has been read
        if (more) stage(next);
      });
      if (!t.is_v) have = page;
      t = next;
      page = page_at(e);
    }
  } else {
    const int32_t per = work.per;
#pragma unroll 1
    for (int32_t c = blockIdx.x - ctas_kv; c < upto[2][kThreads - 1]; c += gridDim.x - ctas_kv) {
      int32_t k = c;
      KvSpan s;
      locate(2, k, s);
      int32_t mine = tid;
      asm volatile("" : "+r"(mine));
      const int64_t e = static_cast<int64_t>(k) * kThreads + mine;
      if (e >= static_cast<int64_t>(s.n) * per) continue;
      const int32_t i = e >> 31 ? static_cast<int32_t>(e / per) : by_part.of(static_cast<int32_t>(e));
      const int32_t ru = static_cast<int32_t>(e - static_cast<int64_t>(i) * per), run = ru / units, u = ru - run * units;
      const RotUnit q = rot_unit(a.rot, u);
      if (!q.turned && a.q == a.q_out) continue;
      rotate_heads(a.q + (s.r0 + i) * a.ldq, a.q_out + (s.r0 + i) * a.ldqo, run * hpt, min(run * hpt + hpt, a.nh), D,
                   a.rot, u, q, s.first + i, false);
    }
  }
}

// ---------------------------------------------------------------- compaction
constexpr int kCompactWarps = 8;

// The float of one e4m3 code.
__device__ __forceinline__ float of_code(uint32_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(c)));
  return __low2float(*reinterpret_cast<const __half2*>(&h));
}

__device__ __forceinline__ uint4 rescale16(uint4 w, __half2 by) {
  return make_uint4(rescale4(w.x, by), rescale4(w.y, by), rescale4(w.z, by), rescale4(w.w, by));
}

// Four codes times a power of two, rounded to codes again (no product passes 448).  In fp32: the power may be any.
__device__ __forceinline__ uint32_t move4(uint32_t codes, float by) {
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(codes >> (16 * i))));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    out |= static_cast<uint32_t>(e4m3x2(f.x * by, f.y * by)) << (16 * i);
  }
  return out;
}

constexpr int kMoves = 256;   // tokens whose places a CTA keeps at a time: two whole pages or more
constexpr float kLeastScale = 0x1p-60f;
constexpr int kInHand = 2;    // passes over a page's tokens that a warp keeps in registers

// A CTA takes a sequence and some of the (cache, keys or values, head) of it, a warp one at a time; where the tokens lie and go
// is found once.  Page by page, so that a token's slot is never written before it has been read: sources rise strictly, so the
// j-th kept token's is j or more behind the context.  A page that has to grow is rounded again before what moves inside it.
// Bound by the chain of loads (rows, path, page numbers, codes and scales), 3 us for one sequence and layer; 16 layers of 64
// sequences with up to 8 moved tokens each (8 heads of 128) move 19.6 MB in 14.4 us where no page grows, and take 18.5 where the
// pages are each at half the scale of the next, so that those that take another's tokens are rounded again.
template <int D>
__global__ void __launch_bounds__(32 * kCompactWarps) kv_compact_kernel(const __grid_constant__ KvCompactArgs a, Divisor by_page,
                                                                        int32_t per_cta) {
  constexpr int kLanes = D / 16, kAtOnce = 32 / kLanes;  // lanes a token, tokens a pass
  __shared__ int32_t src_page[kMoves], src_at[kMoves];    // where the tokens lie: page of the sequence, slot in it
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane / kLanes, word = lane % kLanes;
  const int32_t b = blockIdx.x, page = a.page, heads = 2 * a.nkv, items = a.n_caches * heads;
  const int32_t r0 = a.row_start[b], r1 = a.row_start[b + 1], len = a.seq_len[b], m = a.n_kept[b], n = r1 - r0;
  bool bad = r0 < 0 || r1 < r0 || r1 > a.T || len < 0 || len > static_cast<int64_t>(a.max_pages) * page || m < 0 || m > n;
  // the kept rows rise strictly; the first that is not in its place, all behind it are not either
  int32_t still = 0;
  if (!bad) {
#pragma unroll 1
    for (int32_t j = tid; j < m; j += 32 * kCompactWarps) {
      const int32_t i = a.path[r0 + j];
      bad |= i >= n || i <= (j > 0 ? a.path[r0 + j - 1] : -1);
      still += i == j ? 1 : 0;
    }
  }
  __shared__ int32_t in_place;
  if (tid == 0) in_place = 0;
  if (__syncthreads_or(bad)) {
    if (tid == 0) latch_index_error(a.status);
    return;
  }
  still = __reduce_add_sync(0xffffffffu, still);
  if (lane == 0 && still) atomicAdd(&in_place, still);
  __syncthreads();
  const int32_t first = len - n;
#pragma unroll 1
  for (int32_t c0 = max(in_place, -first), c1; c0 < m; c0 = c1) {  // (slots before the first are not stored)
    // as many tokens as are kept in mind, up to the end of a page
    c1 = m - c0 <= kMoves ? m : by_page.of(first + c0 + kMoves) * page - first;
    __syncthreads();
    for (int32_t j = c0 + tid; j < c1; j += 32 * kCompactWarps) {
      const int32_t at = first + a.path[r0 + j], pg = by_page.of(at);
      src_page[j - c0] = pg;
      src_at[j - c0] = at - pg * page;
    }
    __syncthreads();
#pragma unroll 1
    for (int32_t e = blockIdx.y * per_cta + warp; e < min(items, (static_cast<int32_t>(blockIdx.y) + 1) * per_cta); e += kCompactWarps) {
      const int32_t l = e / heads, hv = e - l * heads, h = hv >= a.nkv ? hv - a.nkv : hv;
      const KvCompactArgs::Cache& kv = a.cache[l];
      uint8_t* const codes = hv >= a.nkv ? kv.v_codes : kv.k_codes;
      float* const scales = hv >= a.nkv ? kv.v_scale : kv.k_scale;
      const int32_t* const table = kv.table + static_cast<int64_t>(b) * a.max_pages;
      auto block_of = [&](int32_t pg) -> int32_t {
        const int32_t id = table[pg];
        if (id >= 0 && id < a.n_pages) return id * a.nkv + h;
        latch_index_error(a.status);
        return -1;
      };
#pragma unroll 1
      for (int32_t j0 = c0, j1; j0 < c1; j0 = j1) {
        const int32_t pg = by_page.of(first + j0);
        j1 = min(c1, (pg + 1) * page - first);
        const int32_t block = block_of(pg);
        uint8_t* const dst = codes + static_cast<int64_t>(max(block, 0)) * page * D;
        const float old = block >= 0 ? scales[block] : 0.0f;
        // a lane's 16 bytes of a token's codes where they lie, its page's scale; whether that is another page
        auto source = [&](int32_t j, uint4& w, float& scale) -> bool {
          const int32_t sp = src_page[j - c0], sb = sp == pg ? block : block_of(sp);
          w = make_uint4(0u, 0u, 0u, 0u);
          scale = old;
          if (sb < 0) return true;
          w = *reinterpret_cast<const uint4*>(codes + (static_cast<int64_t>(sb) * page + src_at[j - c0]) * D + 16 * word);
          if (sp != pg) scale = scales[sb];
          return sp != pg;
        };
        // the scale that a lane's codes under theirs ask for (by the code's and the scale's: their product may pass fp32's range)
        auto wanted = [&](const uint4& q, float scale) {
          constexpr uint32_t kAbs = 0x7f7f7f7fu;
          uint32_t w = __vmaxu4(__vmaxu4(q.x & kAbs, q.y & kAbs), __vmaxu4(q.z & kAbs, q.w & kAbs));
          w = __vmaxu4(w, w >> 16);
          const float s = scale_of(__float_as_uint(of_code(max(w & 0xffu, w >> 8 & 0xffu)))) * scale;
          return s > 0.0f && s < kLeastScale ? kLeastScale : s;
        };
        auto put = [&](int32_t j, const uint4& w) {
          *reinterpret_cast<uint4*>(dst + (first + j - pg * page) * D + 16 * word) = w;
        };
        const int32_t count = j1 - j0;
        const bool in_hand = count <= kInHand * kAtOnce;
        uint4 held[kInHand];
        uint32_t far = 0;  // bit j: the j-th comes from another page
        float from = 0.0f, top = 0.0f;    // (a lane a token: its page's scale)
        if (in_hand) {
          int32_t at = -1;  // its row of codes
          bool other = false;
          if (lane < count) {
            const int32_t sp = src_page[j0 - c0 + lane], sb = block_of(sp);
            other = sp != pg;
            if (sb >= 0) {
              at = sb * page + src_at[j0 - c0 + lane];
              from = scales[sb];
            }
          }
          far = __ballot_sync(0xffffffffu, other);
#pragma unroll
          for (int k = 0; k < kInHand; ++k)
            if (k * kAtOnce < count) {
              const int32_t row = __shfl_sync(0xffffffffu, at, k * kAtOnce + sub);
              held[k] = make_uint4(0u, 0u, 0u, 0u);
              if (row >= 0) held[k] = *reinterpret_cast<const uint4*>(codes + static_cast<int64_t>(row) * D + 16 * word);
            }
#pragma unroll
          for (int k = 0; k < kInHand; ++k)
            if (k * kAtOnce < count) {
              const float scale = __shfl_sync(0xffffffffu, from, k * kAtOnce + sub);
              if (far >> (k * kAtOnce + sub) & 1u)
                asm("max.NaN.f32 %0, %1, %2;" : "=f"(top) : "f"(top), "f"(wanted(held[k], scale)));
            }
        } else {
#pragma unroll 1
          for (int32_t j = j0 + sub; j < j1; j += kAtOnce) {
            uint4 w;
            float scale;
            if (source(j, w, scale)) asm("max.NaN.f32 %0, %1, %2;" : "=f"(top) : "f"(top), "f"(wanted(w, scale)));
          }
        }
        if (block < 0) continue;
        const float want = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu));
        const bool nan = !(want == want) || !(old == old);
        const float now = nan ? __uint_as_float(0x7fffffffu) : fmaxf(old, want);
        const bool grows = !nan && old > 0.0f && now > old;
        const __half2 shrink = __float2half2_rn(grows ? fmaxf(old / now, 5.9604645e-8f) : 1.0f);
        if (lane == 0 && !(now == old)) scales[block] = now;
        if (grows) {
#pragma unroll 1
          for (int32_t k = lane; k < page * D / 16; k += 32) {
            uint4* const at = reinterpret_cast<uint4*>(dst) + k;
            *at = rescale16(*at, shrink);
          }
        }
        auto moved = [&](const uint4& w, float scale) {
          const float by = now > 0.0f ? scale / now : 1.0f;
          return nan ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(move4(w.x, by), move4(w.y, by), move4(w.z, by), move4(w.w, by));
        };
        __syncwarp();
        if (in_hand) {
#pragma unroll
          for (int k = 0; k < kInHand; ++k)
            if (k * kAtOnce < count) {
              const int32_t j = k * kAtOnce + sub;
              const float scale = __shfl_sync(0xffffffffu, from, j);
              if (j < count) put(j0 + j, far >> j & 1u ? moved(held[k], scale) : grows ? rescale16(held[k], shrink) : held[k]);
            }
        } else {
#pragma unroll 1
          for (int32_t j = j0 + sub; __any_sync(0xffffffffu, j < j1); j += kAtOnce) {
            uint4 w;
            float scale;
            if (j < j1 && source(j, w, scale)) w = moved(w, scale);
            __syncwarp();
            if (j < j1) put(j, w);
            __syncwarp();
          }
        }
        __syncwarp();
      }
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
    const int32_t hpt = heads_per_thread(T, nh, d / 16, f32 ? 4 : 8);
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
  const int32_t units = a.cache.d / 16, heads = 2 * a.cache.nkv;
  // (no longer than a sequence's queries fill a chunk: 512 single tokens of 32 heads 14.5 us by runs of 1, 16.9 of 4)
  int32_t hpt = a.q ? heads_per_thread(a.T, a.nh, units, 8) : 1;
  while (hpt > 1 && (a.T + a.B - 1) / a.B * units * ((a.nh + hpt - 1) / hpt) < kThreads) hpt /= 2;
  const int32_t runs = a.q ? (a.nh + hpt - 1) / hpt : 0;
  // Teams of a warp up to 8 tokens a sequence in the mean, of two above (32 / 8 heads of 128: 64 sequences of 1, 8, 12 and 16
  // tokens take 4.5, 5.9, 11.0 and 11.1 us by one warp, 5.7, 7.5, 8.5 and 9.2 by two; four prompts of 2048 in pages of 16
  // tokens 62.7 and 45.9).
  // CTAs for keys and values: as many as there can be work for (a sequence's pages: its rows' and two that it gets a part
  // of), two an SM at most, with queries three for two SMs (32 heads of each, 4 x 1024 tokens: 64 us with one an SM, 45 with
  // 228, 44 with two; 32 / 8 heads, 4 x 2048 tokens: 38, 40 and 40).  The queries' CTAs come behind them, one a chunk up to 304, then
  // for up to four chunks each (the prompts take 40 to 42 us from one to eight).  Any number is right.
  const int64_t team = a.T <= 8 * static_cast<int64_t>(a.B) ? 1 : 2, teams = kThreads / 32 / team;
  const int64_t singles = std::min<int64_t>(a.T, a.B), pages = (a.T - singles) / a.cache.page + (a.T > singles ? singles : 0);
  const int64_t kv = std::min<int64_t>((singles * heads + teams - 1) / teams + pages * heads, a.q ? 228 : 304);
  const int64_t chunks =
      a.q ? std::max((a.T * runs * units + kThreads - 1) / kThreads + (a.T > singles ? singles : 0), singles) : 0;
  const int64_t qs = std::min<int64_t>(std::max<int64_t>(chunks / 4, std::min<int64_t>(chunks, 304)), 1 << 20);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(kv + qs));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr{};  // the kernel waits by itself for the launch ahead
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const auto go = [&](auto d, auto t, auto held) {
    constexpr auto kern = kv_append_kernel<decltype(d)::value, decltype(t)::value, decltype(held)::value>;
    static std::atomic<uint64_t> ready{0};  // devices on which the kernel may use its shared memory
    cfg.dynamicSmemBytes = held * 6 * 16 * kThreads;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = uint64_t(1) << (dev & 63);
    if (!(ready.load(std::memory_order_relaxed) & bit)) {
      e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(cfg.dynamicSmemBytes));
      if (e != cudaSuccess) return e;
      ready.fetch_or(bit, std::memory_order_relaxed);
    }
    return cudaLaunchKernelEx(&cfg, kern, a, static_cast<uint32_t>(kv), hpt, divisor(runs * units), divisor(a.cache.page),
                              divisor(heads));
  };
  constexpr std::integral_constant<int, 1> c1;
  constexpr std::integral_constant<int, 2> c2;
  constexpr std::integral_constant<int, 4> c4;
  constexpr std::integral_constant<int, 64> c64;
  constexpr std::integral_constant<int, 128> c128;
  if (a.cache.d == 64) return team == 1 ? go(c64, c1, c2) : go(c64, c2, c2);
  if (a.cache.page <= 64) return team == 1 ? go(c128, c1, c2) : go(c128, c2, c2);
  return team == 1 ? go(c128, c1, c4) : go(c128, c2, c4);  // pages of 128 tokens of 128 elements
}

cudaError_t launch_kv_compact(KvCompactArgs& a, cudaStream_t st) {
  WaitCtl wc;
  if (!launch_wait_ctl(&wc)) return cudaErrorInvalidDevice;
  a.status = wc.status_word;
  // A warp takes one (cache, keys or values, head) (one layer of one sequence 3.1 us, two each 4.0; 16 layers of 64 sequences
  // 14.4, two each 14.1, four 17.1); as many CTAs a sequence as a grid's second dimension has.
  const int32_t items = a.n_caches * 2 * a.nkv, per_cta = ((items / kCompactWarps) / 65535 + 1) * kCompactWarps;
  const dim3 grid(a.B, (items + per_cta - 1) / per_cta);
  if (a.d == 64)
    kv_compact_kernel<64><<<grid, 32 * kCompactWarps, 0, st>>>(a, divisor(a.page), per_cta);
  else
    kv_compact_kernel<128><<<grid, 32 * kCompactWarps, 0, st>>>(a, divisor(a.page), per_cta);
  return cudaGetLastError();
}

}  // namespace catq
