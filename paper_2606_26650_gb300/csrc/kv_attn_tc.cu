// kv_attn_tc.cu — grouped-query attention of new tokens over the paged cache of 8-bit codes, on the tcgen05
// tensor cores with the codes as they lie in the cache: no element of the cache passes through a register.
//
// With few query rows a key/value head, the cached tokens are the long side: they are the M of both products, the
// rows (new token, query head of the group), R of them a CTA's tile, the N:
//   S^T [128 tokens, 2 R] = K [128, d] Q^T,      O^T [d, 3 R] += V^T [d, 128] P^T [128, 3 R].
// A operands are the code tiles that TMA brings page by page (K K-major, V MN-major: the tensor core transposes it), e4m3
// like the cache.  B operands are 8-bit terms in columns of their own.  Queries are two e4m3 terms, x = hi + lo / 16 with hi =
// e4m3(x), lo = e4m3(16 (x - hi)), 4 + 4 significant bits: a bf16 query (8 bits), scaled by a power of two so that its row's
// largest element lies in (224, 448], is exact but for what is 2^-22 of that element.  (Converting the codes to 16 bits instead
// would cost the CTAs some 4 instructions a pair of elements, at 23 elements a cycle and SM more than the loads themselves.)
//
// The weights of the values are three e5m2 terms, h + m / 8 + l / 64: within 2^-9 of the weight (a bf16 one would be within 2^-8), or
// within 2^-33 of the row's largest, which is 2^10 or more.  That range is needed: one token far above thousands of others is
// ordinary attention, the others count by their sum, and the divisor has all of them.  (Two e4m3 terms, whose floor was 2^-17 of
// the largest, lost a third of the output of 131,071 tokens 2^-18 below one.)
//
// Scores in base 2: x = (S_hi + S_lo / 16) s_k f + log2 s_v for a token of a page with scales s_k, s_v (powers of two) and
// a row whose query's scale and log2(e) / sqrt(d) are in f; weights of the value codes are w = 2^(x - m), the row's sum adds
// w / s_v, and at the end O = O^T / sum, lse = (m + log2 sum) ln 2, both exact for whichever m was used.  m is the row's
// largest x less 10, so that the largest weights are 2^10 and more, and is raised lazily: only when some x - m passes 15.75
// (weights stay below e5m2's largest, 57344) does the group agree on new maxima and rescale its sums and accumulators; a tile is
// scored twice at most.
//
// A CTA has a softmax group of 128 threads for up to 32 rows (16 of heads of 64, whose threads have two tokens; thread t owns
// shared-memory row t of a tile: TMEM lane t), a TMA warp and an MMA warp.  Work: the tiles of all (sequence, key/value head, row
// tile), in this order as one line, each row tile with a head of kHead positions for what its beginning and end cost, cut
// into equal runs, one a CTA, whatever the sequences' lengths are; they are read on the device, so a captured launch
// follows them.  A run that holds only a part of a row tile's tokens leaves its maxima, sums and accumulators in the
// workspace; the last run of the row tile to finish (a counter, which it leaves at zero) joins them in their order, so
// the result does not depend on which one that is.
//
// Bound by the codes' way from HBM where sequences are long: 64 of 300 to 8192 tokens, 32 / 8 heads of 128, one row
// each, take 92 us for 572 MB, 6.2 TB/s (7 while it streams); a build without the softmax's arithmetic takes as
// long, the rest is the start (lengths, page numbers, first tile: 5 us) and the last runs' join.  One sequence of
// 131,071 tokens: 50.3 us for 268 MB.  16 sequences of 1000 to 4500 tokens with 25 rows a head: 30 us for 94 MB, 22 without
// the softmax's arithmetic.  128 sequences of 17 to 2001 tokens, 12 heads of 64: 54 us for 199 MB, 48 without, bound by the
// beginnings and ends of 1536 row tiles.
// Two CTAs an SM: with three (rings of 4 slots) the 64 sequences took 94 us and the long one 54.8, with one (12 slots) 108
// and 51.5, with two 92.5 and 51.8.
//
// Tokens behind a row's own position weigh 0 whatever their scales are; the values behind the last visible token of a tile
// are zeroed in shared memory (what an unfinished page holds there may be anything, NaN codes too).
#include <cuda.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <mutex>

#include "launch.h"
#include "ptx_sm100.cuh"

namespace catq {
namespace {

constexpr int kGroup = 128;                  // threads of a softmax group
constexpr float kNominal = 10.0f;            // log2 of a weight at the maximum taken
constexpr float kOver = 15.75f;              // raise the maximum past this (2^15.75 < 57344)
constexpr float kNoMax = -3e38f;             // maximum of a row that has seen nothing
constexpr uint32_t kLeastScale = (127u - 60u) << 23;  // 2^-60: stands for a scale of 0
constexpr int kLeastExp = -126;              // of a query row's scale: both powers of two, 2^-126 and 2^126, are normal numbers
constexpr float kLoUnit = 0.0625f;           // unit of a query's lo term
constexpr float kUnitM = 0.125f, kUnitL = 0.015625f;  // units of a weight's second and third term
constexpr int kScaleRing = 16;               // tiles whose scales are kept (see the TMA warp)
constexpr int kRows = 128;                   // shared-memory rows of a tile of codes, 128 bytes each

template <int HD, int R>
struct KvLay {
  static constexpr int kHd = HD;
  static constexpr int kR = R;                                       // rows of a row tile
  static constexpr int kTpr = 128 / HD;                              // tokens a shared-memory row
  static constexpr int kTok = kRows * kTpr;                          // cached tokens a tile
  // What a row tile's beginning and end cost, in tiles (one GB300; no such cost: 34 us for drafted tokens, 65 for heads of
  // 64, 53 for one long sequence; with it 30, 54 and 50; 4 for the heads of 64: 59, 1 for the drafted tokens: 33).
  static constexpr int kHead = R == 8 ? (HD == 64 ? 1 : 2) : 4;
  static constexpr int kPages = kTok / 16;                           // most pages a tile
  static constexpr int kCols = 2 * R;                                // N of the scores: two terms of the queries
  static constexpr int kPCols = R == 8 ? 32 : 3 * R;                 // N of the values' product: three terms (of 8 rows: and 8
                                                                     // columns that nothing reads, N is a multiple of 16)
  static constexpr int kMaxChunk = HD == 128 ? 32 : 16;
  static constexpr int kChunk = R < kMaxChunk ? R : kMaxChunk;       // rows of a softmax group
  static constexpr int kGroups = R / kChunk;
  static constexpr int kSoft = kGroups * kGroup;
  static constexpr int kTmaWarp = 4 * kGroups, kMmaWarp = kTmaWarp + 1, kThreads = kSoft + 64;
  static constexpr uint32_t kColO = 2 * kTpr * kCols;                // two buffers of scores, then the accumulators
  static constexpr uint32_t kTmem = kColO + kPCols <= 64 ? 64 : kColO + kPCols <= 128 ? 128 : kColO + kPCols <= 256 ? 256 : 512;
  static constexpr int kCtas = kTmem <= 256 ? 2 : 1;                 // CTAs an SM
  static constexpr uint32_t kTile = kRows * 128;                     // a tile of codes
  static constexpr uint32_t kQ = kCols * HD, kP = kTok * kPCols;
  // barriers, tensor-memory address, start of the run | scales of the tiles in flight | per row: query factor, maximum,
  // its last raise, last position, output offset (8 bytes), sums by warp | Q, P twice, ring
  static constexpr uint32_t kOffScale = 640, kOffF = kOffScale + kScaleRing * 8 * kPages, kOffM = kOffF + 4 * R,
                            kOffFac = kOffM + 4 * R, kOffLim = kOffFac + 4 * R, kOffRow = kOffLim + 4 * R,
                            kOffZero = kOffRow + 8 * R, kOffRed = kOffZero + 4 * R,
                            kOffQ = (kOffRed + 16 * R + 127) / 128 * 128, kOffP = kOffQ + kQ,
                            kOffRing = (kOffP + 2 * kP + 1023) / 1024 * 1024;
  static constexpr uint32_t kBudget = (kCtas == 2 ? 112 : 224) * 1024;
  static constexpr int kSlots0 = (kBudget - 1024 - kOffRing) / kTile;
  static constexpr int kSlots = kSlots0 > 12 ? 12 : kSlots0;
  static constexpr uint32_t kBarFull = 0, kBarEmpty = 8 * kSlots, kBarScale = 16 * kSlots, kBarRest = kBarScale + 8 * kScaleRing;
  static constexpr uint32_t kSmem = kOffRing + kSlots * kTile + 1024;
  static constexpr int kPartFloats = R * (HD + 2);                   // maxima, sums, accumulators of a part
};

// ---------------------------------------------------------------- the line of tiles
// One sequence's share of the line: `per_head` positions for each key/value head.  Every row tile has a stretch of kHead
// positions and one for each of its tiles: runs of equal length are then runs of nearly equal time.
struct KvSeq {
  int32_t r0, n, len;  // first row, rows, cached tokens
  int64_t per_head;
};

struct KvGeom {
  const int32_t *row_start, *seq_len;
  int32_t B, group, nkv;
  uint32_t group_inv;  // ceil(2^32 / group): rows below 2^26 are divided by one product
  int64_t T, max_len;
  __device__ __forceinline__ int32_t token_of(int32_t row) const {
    return group == 1 ? row : static_cast<int32_t>(__umulhi(static_cast<uint32_t>(row), group_inv));
  }
};

// Tokens that the row tile `q` of a sequence can see.
template <class Y>
__device__ __forceinline__ int32_t visible(const KvGeom& g, const KvSeq& s, int32_t q) {
  return max(s.len - s.n + g.token_of(min((q + 1) * Y::kR, s.n * g.group) - 1) + 1, 0);
}
template <class Y>
__device__ __forceinline__ int32_t row_tiles(const KvGeom& g, const KvSeq& s) {
  return (s.n * g.group + Y::kR - 1) / Y::kR;
}
// A row tile that sees nothing still has a tile: its rows are written.
template <class Y>
__device__ __forceinline__ int32_t tiles_of(int32_t vis) { return max((vis + Y::kTok - 1) / Y::kTok, 1); }

template <class Y>
__device__ __forceinline__ KvSeq load_seq(const KvGeom& g, int32_t b, int32_t* status) {
  KvSeq s;
  s.r0 = g.row_start[b];
  const int32_t r1 = g.row_start[b + 1];
  s.len = g.seq_len[b];
  s.n = r1 - s.r0;
  s.per_head = 0;
  if (s.r0 < 0 || r1 < s.r0 || r1 > g.T || s.len < 0 || s.len > g.max_len) {
    if (status) atomicCAS(status, 0, 10 /* CATQ_ERR_INDEX */);
    s.n = 0;
    return s;
  }
  const int32_t nq = row_tiles<Y>(g, s);
#pragma unroll 1
  for (int32_t q = 0; q < nq; ++q) s.per_head += Y::kHead + tiles_of<Y>(visible<Y>(g, s, q));
  return s;
}

// Walks a run's segments: a segment is the run's part of one row tile.
template <class Y>
struct KvWalk {
  int64_t at, end;       // line positions still to do
  int32_t b, h, q, t;    // the next position: sequence, head, row tile, place in the row tile's stretch
  KvSeq s;
  // the segment
  int32_t n;             // its tiles
  int32_t t0;            // first of them
  int32_t all, vis;      // the row tile's tiles and visible tokens
  int64_t begin;         // line position of the row tile's first tile
  int32_t sb, sh, sq;    // its sequence, head, row tile
  int32_t r0, rows_n, len;  // its sequence's first row, rows, cached tokens
  __device__ __forceinline__ bool next(const KvGeom& g) {
    for (;;) {
      if (at >= end) return false;
      if (s.per_head == 0 || h == g.nkv) {
#pragma unroll 1
        do {
          if (++b >= g.B) return false;  // (the lengths changed under the kernel)
          s = load_seq<Y>(g, b, nullptr);
        } while (s.per_head == 0);
        h = q = t = 0;
      }
      sb = b; sh = h; sq = q; r0 = s.r0; rows_n = s.n; len = s.len;
      vis = visible<Y>(g, s, q);
      all = tiles_of<Y>(vis);
      const int32_t part = static_cast<int32_t>(min(static_cast<int64_t>(Y::kHead + all - t), end - at));
      begin = at - t + Y::kHead;
      t0 = max(t - Y::kHead, 0);
      n = t + part - Y::kHead - t0;
      at += part;
      t = 0;
      if (++q == row_tiles<Y>(g, s)) {
        q = 0;
        ++h;
      }
      if (n > 0) return true;  // (a run that ends in a row tile's head leaves it to the next)
    }
  }
};

// ---------------------------------------------------------------- operands
__device__ __forceinline__ float fast_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Two values (|x| <= 448) as hi + lo / 16: two e4m3 numbers each.  Through fp16, whose 11 bits are more than both terms'.
__device__ __forceinline__ void split2(float x0, float x1, uint16_t& hi, uint16_t& lo) {
  uint32_t h16, back;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h16) : "f"(x1), "f"(x0));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(hi) : "r"(h16));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(hi));
  const __half2 rest = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&h16), *reinterpret_cast<const __half2*>(&back)),
                               __float2half2_rn(16.0f));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(lo) : "r"(*reinterpret_cast<const uint32_t*>(&rest)));
}

// Four weights, rounded to fp16, as words of three e5m2 terms, h + m / 8 + l / 64 (SCALED) or h + m + l.  e5m2 is fp16's upper byte:
// a term is a mask, after half a step's addition where it is rounded, and what it leaves is exact in fp16.  Weights up to 2^15.75,
// where no term passes e5m2's largest: within 2^-9 of the weight, or 2^-23 (SCALED), 2^-17.  h is rounded so that m and l have
// either sign: added to one accumulator, which cuts off what is below its last bit, they would lose part of a one-sided sum
// (h cut off too, 2^19 tokens of equal weight: the output 0.4 % too small instead of 0.08 %).  m is cut off, an instruction a
// pair less.
template <bool SCALED>
__device__ __forceinline__ void split3(const float* x, uint32_t& h, uint32_t& m, uint32_t& l) {
  uint32_t a[2], b[2], c[2];
  const auto rest = [](uint32_t v, uint32_t term, float unit) {
    term &= 0xff00ff00u;
    __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&term));
    if (SCALED) r = __hmul2(r, __float2half2_rn(unit));
    return *reinterpret_cast<const uint32_t*>(&r);
  };
  constexpr uint32_t kHalfStep = 0x00800080u;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    a[i] = w + kHalfStep;
    b[i] = rest(w, a[i], 1.0f / kUnitM);
    c[i] = rest(b[i], b[i], kUnitM / kUnitL) + kHalfStep;
  }
  h = __byte_perm(a[0], a[1], 0x7531);
  m = __byte_perm(b[0], b[1], 0x7531);
  l = __byte_perm(c[0], c[1], 0x7531);
}

// Eight values as eight bytes of either term.
__device__ __forceinline__ void split8(const float* x, uint2& hi, uint2& lo) {
  uint16_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) split2(x[2 * i], x[2 * i + 1], h[i], l[i]);
  hi = make_uint2(h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16);
  lo = make_uint2(l[0] | static_cast<uint32_t>(l[1]) << 16, l[2] | static_cast<uint32_t>(l[3]) << 16);
}

// Upper half of a shared-memory matrix descriptor: the stride, the descriptor's version, the swizzle (0 none, 2 128-byte,
// 4 64-byte rows).
__host__ __device__ constexpr uint32_t desc_hi(uint32_t sbo, uint32_t swizzle) { return (sbo >> 4) | (1u << 14) | (swizzle << 29); }

__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi,
                                        uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %5, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Instruction descriptor of kind::f8f6f4: A and B e4m3 or, if said, e5m2, fp32 D.
__host__ __device__ constexpr uint32_t idesc_f8(uint32_t M, uint32_t N, bool a_mn, bool b_mn, bool a_e5m2 = false,
                                                bool b_e5m2 = false) {
  return (1u << 4) | ((a_e5m2 ? 1u : 0u) << 7) | ((b_e5m2 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) |
         ((b_mn ? 1u : 0u) << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// N rows' products (8 where R is, else 16) from their hi columns at `base` and their lo columns R behind: hi + lo / 16, by
// pairs.
template <int R, int N>
__device__ __forceinline__ void load_rows(uint32_t base, float2 (&t)[N / 2]) {
  uint32_t v[2 * N];
  if constexpr (N == R && N == 8) {
    tmem_ld16(base, v);
  } else {
    tmem_ld16(base, *reinterpret_cast<uint32_t(*)[16]>(&v[0]));
    tmem_ld16(base + R, *reinterpret_cast<uint32_t(*)[16]>(&v[N]));
  }
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < N / 2; ++i)
    t[i] = fma2(make_float2(__uint_as_float(v[N + 2 * i]), __uint_as_float(v[N + 2 * i + 1])), both(kLoUnit),
                make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])));
}
// N rows' sums (8 where R is, else 16) from their three terms' accumulators, R columns apart, by pairs.
template <int R, int N>
__device__ __forceinline__ void load_sums(uint32_t base, float2 (&t)[N / 2]) {
  uint32_t v[3 * N];
  if constexpr (N == R && N == 8) {
    tmem_ld16(base, *reinterpret_cast<uint32_t(*)[16]>(&v[0]));
    tmem_ld8(base + 16, *reinterpret_cast<uint32_t(*)[8]>(&v[16]));
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k) tmem_ld16(base + k * R, *reinterpret_cast<uint32_t(*)[16]>(&v[k * N]));
  }
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const auto term = [&](int k) {
      return make_float2(__uint_as_float(v[k * N + 2 * i]), __uint_as_float(v[k * N + 2 * i + 1]));
    };
    t[i] = fma2(term(2), both(kUnitL), fma2(term(1), both(kUnitM), term(0)));
  }
}
// Eight columns at `base`, and those `step` behind them N times, times f.
template <int N>
__device__ __forceinline__ void scale_cols8(uint32_t base, int step, const float2 (&f)[4]) {
  uint32_t v[N][8];
#pragma unroll
  for (int k = 0; k < N; ++k) tmem_ld8(base + k * step, v[k]);
  tmem_ld_wait();
#pragma unroll
  for (int k = 0; k < N; ++k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 w = mul2(make_float2(__uint_as_float(v[k][2 * i]), __uint_as_float(v[k][2 * i + 1])), f[i]);
      v[k][2 * i] = __float_as_uint(w.x);
      v[k][2 * i + 1] = __float_as_uint(w.y);
    }
    tmem_st8(base + k * step, v[k]);
  }
}

__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Sums (or maxima) over a warp of v[0 .. CH), CH <= 32: afterwards v[0] of lane l holds that of row l / (32 / CH).
template <int CH, bool MAX>
__device__ __forceinline__ void warp_rows(float (&v)[CH], int lane) {
  int n = CH;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (n > 1) {
      n /= 2;
      const bool up = (lane & o) != 0;
#pragma unroll
      for (int i = 0; i < CH / 2; ++i)
        if (i < n) {
          const float send = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
          const float got = __shfl_xor_sync(0xffffffffu, send, o);
          v[i] = MAX ? fmaxf(keep, got) : keep + got;
        }
    } else {
      const float got = __shfl_xor_sync(0xffffffffu, v[0], o);
      v[0] = MAX ? fmaxf(v[0], got) : v[0] + got;
    }
  }
}

// N floats of shared memory (16-byte aligned) by pairs.
template <int N>
__device__ __forceinline__ void load_row(const float* p, float2 (&v)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float4 a = reinterpret_cast<const float4*>(p)[i];
    v[2 * i] = make_float2(a.x, a.y);
    v[2 * i + 1] = make_float2(a.z, a.w);
  }
}

__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
  const uint64_t t0 = globaltimer_ns();
  while (!mbar_try_wait(bar, parity))
    if (globaltimer_ns() - t0 > 200000000ull) return;
}

struct KvTcArgs {
  KvAttnArgs a;
  KvGeom g;
  uint32_t* counters;  // [gridDim.x]
  float* parts;        // [gridDim.x][2][kPartFloats]
  WaitCtl wc;
};

// The run of this CTA: every CTA adds up all sequences' tiles, a thread a stretch of them.  A run is at least a row tile of two
// tiles, or of one where no sequence has more (prompts of 64 and 100 tokens, 32 / 8 heads of 128: 15.3 and 15.7 us with two,
// 9.8 and 10.2 with one).  scan [warps], longest [warps] and start [4]: shared memory.  Every thread of the CTA comes here,
// and what it wrote before is visible to all afterwards, tensor memory's address too.
template <class Y>
__device__ __forceinline__ KvWalk<Y> find_run(const KvTcArgs& p, int64_t* scan, int32_t* longest, int32_t* start, int64_t& run,
                                              int64_t& first) {
  const KvGeom& g = p.g;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t total;
  {
    const int32_t per = (g.B + Y::kThreads - 1) / Y::kThreads;
    const int32_t b0 = min(static_cast<int32_t>(threadIdx.x) * per, g.B), b1 = min(b0 + per, g.B);
    int64_t mine = 0;
    int32_t most = 1;
#pragma unroll 1
    for (int32_t b = b0; b < b1; ++b) {
      const KvSeq s = load_seq<Y>(g, b, blockIdx.x == 0 ? p.a.status : nullptr);
      mine += s.per_head * g.nkv;
      if (s.n > 0) most = max(most, tiles_of<Y>(s.len));
    }
    most = __reduce_max_sync(0xffffffffu, most);
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) {
      scan[warp] = upto;
      longest[warp] = most;
    }
    __syncthreads();
    total = 0;
#pragma unroll 1
    for (int w = 0; w < Y::kThreads / 32; ++w) {
      if (w < warp) upto += scan[w];
      total += scan[w];
      most = max(most, longest[w]);
    }
    run = max((total + gridDim.x - 1) / gridDim.x, static_cast<int64_t>(Y::kHead + min(most, 2)));
    first = run * blockIdx.x;
    if (upto - mine <= first && first < upto) {  // the thread whose stretch holds the run's first tile
      int64_t rest = first - (upto - mine);
      int32_t b = b0;
      KvSeq s = load_seq<Y>(g, b, nullptr);
#pragma unroll 1
      while (rest >= s.per_head * g.nkv && b + 1 < b1) {
        rest -= s.per_head * g.nkv;
        s = load_seq<Y>(g, ++b, nullptr);
      }
      const int32_t h = static_cast<int32_t>(rest / max(s.per_head, static_cast<int64_t>(1)));
      rest -= h * s.per_head;
      int32_t q = 0;
#pragma unroll 1
      for (int32_t n; q < row_tiles<Y>(g, s) - 1 && rest >= (n = Y::kHead + tiles_of<Y>(visible<Y>(g, s, q))); ++q) rest -= n;
      start[0] = b;
      start[1] = h;
      start[2] = q;
      start[3] = static_cast<int32_t>(rest);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  KvWalk<Y> w;
  w.at = first;
  w.end = min(first + run, total);
  if (w.at < w.end) {
    w.b = start[0];
    w.h = start[1];
    w.q = start[2];
    w.t = start[3];
    w.s = load_seq<Y>(g, w.b, nullptr);
  }
  return w;
}

// The copying warp of a CTA: every tile of its run through the ring of NS slots.
template <class Y>
__device__ __forceinline__ void copy_tiles(const CUtensorMap& tmk, const CUtensorMap& tmv, const KvTcArgs& p, KvWalk<Y> w,
                                           uint32_t base, float* scales) {
  constexpr int NS = Y::kSlots, kTok = Y::kTok, TPR = Y::kTpr, HD = Y::kHd;
  const uint32_t full0 = base + Y::kBarFull, empty0 = base + Y::kBarEmpty, scale_full0 = base + Y::kBarScale;
  const int lane = threadIdx.x & 31;
  const KvGeom& g = p.g;
  const KvCacheDev& kv = p.a.cache;
  const int32_t ppt = kTok / kv.page;  // pages a tile
  bool ok = true;
  int slot = 0, loads = 0;
  uint32_t ph = 1, gt = 0;
  // A lane a page: the lane's page in tile t of the segment (first row of its block, -1: none), its scales.  Ordinary loads: the
  // launch ahead may have written scales and table while this kernel was resident already, and a non-coherent load (ld.global.nc)
  // is only defined for what no one writes while the kernel lives.
  struct Page {
    int32_t row;
    float ks, vs;
  };
  auto page_of = [&](int32_t j) -> int32_t {
    const int32_t tok = (w.t0 + j) * kTok + lane * kv.page;
    if (j >= w.n || lane >= ppt || tok >= w.vis) return -1;
    return kv.table[static_cast<int64_t>(w.sb) * kv.max_pages + tok / kv.page];
  };
  auto block_of = [&](int32_t j, int32_t id) {
    Page g{-1, 0.0f, 0.0f};
    if (j >= w.n || lane >= ppt || (w.t0 + j) * kTok + lane * kv.page >= w.vis) return g;
    if (id < 0 || id >= kv.n_pages) {
      atomicCAS(p.a.status, 0, 10 /* CATQ_ERR_INDEX */);
      g.row = kv.n_pages * kv.nkv * (kv.page / TPR);  // behind the last row: zeros
      return g;
    }
    const int32_t block = id * kv.nkv + w.sh;
    g.row = block * (kv.page / TPR);
    g.ks = kv.k_scale[block];
    g.vs = kv.v_scale[block];
    return g;
  };
  // A tile into the next slot; with its keys go its scales, into a ring of kScaleRing tiles of their own.  That is
  // deep enough without an empty barrier: while a tile's scales are read its values hold their slot, and the NS slots
  // from there on hold the keys of at most NS / 2 + 3 further tiles.
  static_assert(NS / 2 + 4 <= kScaleRing, "ring of scales");
  auto load = [&](const CUtensorMap* map, const Page& g, bool keys) -> bool {
    const uint32_t pages = __popc(__ballot_sync(0xffffffffu, g.row >= 0));
    if (!mbar_wait_warp(empty0 + 8u * slot, ph, p.wc)) return false;
    if (lane == 0) mbar_arrive_expect_tx(full0 + 8u * slot, pages * kv.page * HD);
    __syncwarp();
    if (g.row >= 0)
      tma_load_2d(base + Y::kOffRing + slot * Y::kTile + lane * kv.page * HD, map, full0 + 8u * slot, 0, g.row);
    if (keys) {
      if (lane < Y::kPages) {
        float* const to = scales + (gt % kScaleRing) * (2 * Y::kPages);
        to[lane] = g.ks;
        to[Y::kPages + lane] = g.vs;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive_local(scale_full0 + 8u * (gt % kScaleRing));
      ++gt;
    }
    ++loads;
    if (++slot == NS) { slot = 0; ph ^= 1u; }
    return true;
  };
  while (ok && w.next(g)) {
    // In the order in which the products take them: K0 K1 V0 K2 V1 ...; a tile's page number is asked for two tiles
    // ahead and its scales one, so that only a segment's first wait for memory.
    const int32_t id0 = page_of(0), id1 = page_of(1);
    int32_t id = page_of(2);
    Page g0 = block_of(0, id0), g1 = block_of(1, id1), g2{-1, 0.0f, 0.0f};
    ok = load(&tmk, g0, true) && (w.n < 2 || load(&tmk, g1, true));
    for (int32_t j = 0; ok && j < w.n; ++j) {
      g2 = block_of(j + 2, id);
      id = page_of(j + 3);
      ok = load(&tmv, g0, false) && (j + 2 >= w.n || load(&tmk, g2, true));
      g0 = g1;
      g1 = g2;
    }
  }
  // copies still in flight land before the CTA exits
#pragma unroll 1
  for (int t = max(0, loads - NS); t < loads; ++t) drain(full0 + 8u * (t % NS), (t / NS) & 1);
}

template <int HD, int R>
__global__ void __launch_bounds__(KvLay<HD, R>::kThreads, KvLay<HD, R>::kCtas)
    kv_attn_kernel(const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv, const KvTcArgs p) {
  using Y = KvLay<HD, R>;
  constexpr int NC = Y::kCols, PC = Y::kPCols, CH = Y::kChunk, NS = Y::kSlots, kThreads = Y::kThreads, kSoft = Y::kSoft,
                kTok = Y::kTok, TPR = Y::kTpr;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* const gbase = smem_raw + (base - raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full0 = base + Y::kBarFull, empty0 = base + Y::kBarEmpty, scale_full0 = base + Y::kBarScale,
                 s_full0 = base + Y::kBarRest, p_full0 = s_full0 + 16, pv_done0 = p_full0 + 16, q_full = pv_done0 + 16,
                 final_bar = q_full + 8;
  static_assert(Y::kBarRest + 3 * 16 + 2 * 8 <= 400, "barriers");
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(gbase + 400);
  int32_t* const merge_flag = reinterpret_cast<int32_t*>(gbase + 404);
  int32_t* const start = reinterpret_cast<int32_t*>(gbase + 408);           // b, h, q, t of the run's first tile
  int64_t* const scan = reinterpret_cast<int64_t*>(gbase + 424);            // warps' sums
  int32_t* const longest = reinterpret_cast<int32_t*>(gbase + 424 + 8 * (kThreads / 32));  // warps' longest sequences, in tiles
  static_assert(424 + 12 * (kThreads / 32) <= Y::kOffScale, "start");
  float* const scales = reinterpret_cast<float*>(gbase + Y::kOffScale);     // [kScaleRing][key scales, value scales of kPages]
  float* const row_f = reinterpret_cast<float*>(gbase + Y::kOffF);
  float* const row_m = reinterpret_cast<float*>(gbase + Y::kOffM);
  float* const row_fac = reinterpret_cast<float*>(gbase + Y::kOffFac);
  int32_t* const row_lim = reinterpret_cast<int32_t*>(gbase + Y::kOffLim);
  int64_t* const row_at = reinterpret_cast<int64_t*>(gbase + Y::kOffRow);
  float* const row_zero = reinterpret_cast<float*>(gbase + Y::kOffZero);
  float* const red = reinterpret_cast<float*>(gbase + Y::kOffRed);          // [groups][4][CH]

  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(full0 + 8u * i, 1);
      mbar_init(empty0 + 8u * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full0 + 8u * i, 1);
      mbar_init(p_full0 + 8u * i, kSoft / 32);
      mbar_init(pv_done0 + 8u * i, 1);
    }
    for (int i = 0; i < kScaleRing; ++i) mbar_init(scale_full0 + 8u * i, 1);
    mbar_init(q_full, kSoft / 32);
    mbar_init(final_bar, 1);
    fence_mbar_init_cluster();
  }
  if (warp == Y::kMmaWarp) tmem_alloc<1>(smem_u32(tmem_slot), Y::kTmem);
  if (warp == Y::kTmaWarp && lane == 0) {
    prefetch_tmap(&tmk);
    prefetch_tmap(&tmv);
  }
  // so far nothing that the launch ahead may have written was read
  grid_launch_dependents();
  grid_dependency_wait();

  const KvGeom& g = p.g;
  int64_t run, first;
  KvWalk<Y> w = find_run<Y>(p, scan, longest, start, run, first);
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t kColO = Y::kColO;
  const KvCacheDev& kv = p.a.cache;
  bool ok = true;

  if (warp == Y::kTmaWarp) {
    copy_tiles<Y>(tmk, tmv, p, w, base, scales);
  } else if (warp == Y::kMmaWarp) {
    constexpr uint32_t idesc_s = idesc_f8(kRows, NC, false, false), idesc_o = idesc_f8(HD, PC, true, true, false, true);
    constexpr uint32_t kHi = desc_hi(1024, 2);  // code tiles: 8 swizzled rows of 128 bytes from one group to the next
    constexpr uint32_t kHiQ = desc_hi(128, 0), kHiP = desc_hi(16 * kRows, 0);
    const bool issuer = elect_one();
    int slot = 0;
    uint32_t ph = 0, gt = 0, seg = 0;  // gt: tiles so far
    auto step = [&] {
      if (++slot == NS) { slot = 0; ph ^= 1u; }
    };
    auto issue_s = [&](uint32_t buf) -> bool {
      if (!mbar_wait_warp(full0 + 8u * slot, ph, p.wc)) return false;
      tc_fence_after();
      if (issuer) {
        const uint32_t ad = desc_lo(base + Y::kOffRing + slot * Y::kTile, 16), bd = desc_lo(base + Y::kOffQ, 16 * NC);
#pragma unroll
        for (int k = 0; k < 4; ++k)  // 32 bytes of a row: HD / 32 steps a token
          umma_f8(tmem + buf * (TPR * NC) + k / (HD / 32) * NC, ad + 2 * k, kHi, bd + 2 * NC * (k % (HD / 32)), kHiQ, idesc_s,
                  k % (HD / 32) > 0 ? 1u : 0u);
        umma_commit<1>(s_full0 + 8u * buf);
        umma_commit<1>(empty0 + 8u * slot);
      }
      step();
      return true;
    };
    while (ok && w.next(g)) {
      if (!mbar_wait_warp(q_full, seg & 1, p.wc) || !issue_s(gt & 1) || (w.n > 1 && !issue_s((gt + 1) & 1))) {
        ok = false;
        break;
      }
      ++seg;
      for (int32_t j = 0; j < w.n; ++j, ++gt) {
        const uint32_t buf = gt & 1;
        if (!mbar_wait_warp(full0 + 8u * slot, ph, p.wc) || !mbar_wait_warp(p_full0 + 8u * buf, (gt >> 1) & 1, p.wc)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (issuer) {
          const uint32_t ad = desc_lo(base + Y::kOffRing + slot * Y::kTile, 16),
                         bd = desc_lo(base + Y::kOffP + buf * Y::kP, 128);
#pragma unroll
          for (int k = 0; k < 4 * TPR; ++k)  // 32 rows, one token of each at a time
            umma_f8(tmem + kColO, ad + 256 * (k % 4) + 4 * (k / 4), kHi, bd + 32 * (k % 4) + 8 * PC * (k / 4), kHiP, idesc_o,
                    (j > 0 || k > 0) ? 1u : 0u);
          umma_commit<1>(pv_done0 + 8u * buf);
          umma_commit<1>(empty0 + 8u * slot);
        }
        step();
        if (j + 2 < w.n && !issue_s(buf)) { ok = false; break; }
      }
    }
    if (issuer) umma_commit<1>(final_bar);
    __syncwarp();
    drain(final_bar, 0);  // every MMA has completed before TMEM is released
  } else {
    // softmax: group wg has rows CH wg .. of the row tile, thread tid of it the tokens of row tid of every tile
    const int wg = warp >> 2, tid = threadIdx.x & (kGroup - 1), bar = 1 + wg, bar_every = 1 + Y::kGroups;
    const int r0 = CH * wg;
    const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + r0;
    float* const my_red = red + wg * 4 * CH;
    const int page_at = TPR * tid / kv.page;
    uint32_t gt = 0, ring = 0;  // tiles and loads before the segment's
    // Products with the values up to tile t of the run have completed.  A barrier for every other tile: the scores of
    // tile t that the caller has seen followed the product of tile t - 2, so the barrier is at most one phase behind,
    // where a single one could be two behind and show the awaited parity.
    auto wait_pv = [&](uint32_t t) { return mbar_wait_warp(pv_done0 + 8u * (t & 1), (t >> 1) & 1, p.wc); };
    // Queries, HD / 8 threads a row: a segment's are asked for while the segment before it is under way.
    constexpr int kPerRow = HD / 8, kPass = kGroup / kPerRow, kPasses = (CH + kPass - 1) / kPass;
    uint4 raw[kPasses];
    auto ask = [&](const KvWalk<Y>& v) {
#pragma unroll
      for (int k = 0; k < kPasses; ++k) {
        const int r = k * kPass + tid / kPerRow, row = v.sq * R + r0 + r;
        raw[k] = make_uint4(0u, 0u, 0u, 0u);
        if (r < CH && row < v.rows_n * g.group) {
          const int32_t tk = g.token_of(row);
          raw[k] = *reinterpret_cast<const uint4*>(p.a.q + (v.r0 + tk) * p.a.ldq +
                                                   (v.sh * g.group + row - tk * g.group) * HD + 8 * (tid % kPerRow));
        }
      }
    };
    constexpr bool kAhead = CH <= 16;  // (32 rows a group: the registers are needed, and a segment is mostly long)
    bool more = w.next(g);
    if (kAhead && more) ask(w);
    KvWalk<Y> ahead;
#pragma unroll 1
    for (; more; w = ahead) {
      if (!bar_all(bar_every, kSoft, ok)) { ok = false; break; }  // the rows' arrays are free
      const int32_t rows = min(R, w.rows_n * g.group - w.sq * R);
      const bool active = r0 < rows;
      if (active) {
        if (!kAhead) ask(w);
        const int i = tid % kPerRow;
        if (tid < CH) {
          const int row = w.sq * R + r0 + tid;
          const int32_t tk = g.token_of(row);
          row_m[r0 + tid] = kNoMax;
          row_zero[r0 + tid] = 0.0f;
          row_lim[r0 + tid] = r0 + tid < rows ? w.len - w.rows_n + tk : -1;
          row_at[r0 + tid] = (w.r0 + tk) * p.a.ldo + (w.sh * g.group + row - tk * g.group) * HD;
        }
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
          const int r = k * kPass + tid / kPerRow;
          const uint32_t u[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
          float x[8];
          uint32_t top = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(u[e] << 16);
            x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
            top = max(top, max(u[e] << 16 & 0x7fffffffu, u[e] & 0x7fff0000u));
          }
#pragma unroll
          for (int o = 1; o < kPerRow; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
          // 2^-e brings the largest element into (224, 448]; a row that is not finite has NaN as its factor
          const int e = max(static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), kLeastExp);
          const bool bad = top >= 0x7f800000u;
          const float by = bad ? 0.0f : __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
          for (int q = 0; q < 8; ++q) x[q] = bad ? 0.0f : x[q] * by;
          uint2 hi, lo;
          split8(x, hi, lo);
          if (r < CH) {
            // K-major without swizzle: 16 bytes of a row, the next 7 rows, the next rows' groups; then the next 16 bytes
            uint8_t* const at = gbase + Y::kOffQ + (i / 2) * (16 * NC) + (r0 + r) * 16 + (i % 2) * 8;
            *reinterpret_cast<uint2*>(at) = hi;
            *reinterpret_cast<uint2*>(at + 16 * R) = lo;
            if (i == 0)
              row_f[r0 + r] = bad ? __uint_as_float(0x7fffffffu)
                                  : __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * p.a.scale_log2;
          }
        }
        fence_proxy_async_smem();
      }
      bar_sync(bar, kGroup);
      if (lane == 0) mbar_arrive_local(q_full);
      ahead = w;
      more = ahead.next(g);
      if (kAhead && more) ask(ahead);
      // tokens that the group's first row sees (the others at least as many)
      const int32_t sees_all = active ? row_lim[r0] + 1 : 0;
      float l[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) l[i] = 0.0f;

      bool failed = false;
#pragma unroll 1
      for (int32_t j = 0; j < w.n; ++j, ++gt) {
        const uint32_t buf = gt & 1;
        if (!active) {  // rows behind the last: the group only keeps pace
          ok = mbar_wait_warp(s_full0 + 8u * buf, (gt >> 1) & 1, p.wc) && ok;
          if (!bar_all(bar, kGroup, ok)) { failed = true; break; }
          if (lane == 0) mbar_arrive_local(p_full0 + 8u * buf);
          continue;
        }
        ok = mbar_wait_warp(scale_full0 + 8u * (gt % kScaleRing), (gt / kScaleRing) & 1, p.wc) && ok;
        const float* const at_scale = scales + (gt % kScaleRing) * (2 * Y::kPages) + page_at;
        float ks = at_scale[0];
        uint32_t vb = __float_as_uint(at_scale[Y::kPages]);
        // log2 and reciprocal of the values' scale; codes under a scale of 0 are zeros, any scale serves them, and the least
        // that an append writes leaves the row's maximum to the pages that have values; one that is not finite makes the scores
        // of the rows that see the token NaN
        if (vb == 0u) vb = kLeastScale;
        if (vb >= 0x7f800000u) {
          ks = __uint_as_float(0x7fffffffu);
          vb = 127u << 23;
        }
        const float lsv = static_cast<float>(static_cast<int>(vb >> 23) - 127);
        const float inv = __uint_as_float((254u - (vb >> 23)) << 23);
        const int32_t tile = (w.t0 + j) * kTok;
        const bool masked = tile + kTok > sees_all;
        ok = mbar_wait_warp(s_full0 + 8u * buf, (gt >> 1) & 1, p.wc) && ok;
        tc_fence_after();
        if (wg == 0 && tile + kTok > w.vis) {
          // the values behind the last visible token become zeros
          const uint32_t at = ring + min(2, w.n) + j + max(0, min(j, w.n - 2)), sl = at % NS;
          ok = mbar_wait_warp(full0 + 8u * sl, (at / NS) & 1, p.wc) && ok;
          uint4* const v = reinterpret_cast<uint4*>(gbase + Y::kOffRing + sl * Y::kTile);
          for (int32_t i = max(w.vis - tile, 0) / TPR * 8 + tid; i < kRows * 8; i += kGroup)  // (chunks of a row are swizzled)
            if (tile + TPR * (i / 8) + ((i ^ (i / 8)) & 7) / (HD / 16) >= w.vis) v[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        // element e CH + i: token e of the thread's, row i of the group's
        float y[TPR * CH];
        constexpr int kStep = CH < 16 ? 8 : 16;
        const int tok = tile + TPR * tid;
        // x as it is rounded, then less the maximum, so that a weight is at most 2^kNominal after a raise however large the
        // scores are (a fused x - m could exceed it by the rounding of x)
        auto score = [&](const float* less) {
#pragma unroll
          for (int c = 0; c < CH; c += kStep) {
            float2 t[kStep / 2], f[kStep / 2], m[kStep / 2];
            load_row<kStep>(row_f + r0 + c, f);
            load_row<kStep>(less + r0 + c, m);
#pragma unroll
            for (int i = 0; i < kStep / 2; ++i) f[i] = mul2(both(ks), f[i]);
#pragma unroll
            for (int e = 0; e < TPR; ++e) {
              load_rows<R, kStep>(lanes + buf * (TPR * NC) + e * NC + c, t);
#pragma unroll
              for (int i = 0; i < kStep / 2; ++i) {
                const float2 v = fma2(m[i], both(-1.0f), fma2(t[i], f[i], both(lsv)));
                y[e * CH + c + 2 * i] = v.x;
                y[e * CH + c + 2 * i + 1] = v.y;
              }
            }
          }
          if (masked) {
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
              for (int e = 0; e < TPR; ++e)
                if (tok + e > row_lim[r0 + i]) y[e * CH + i] = -INFINITY;
          }
        };
        // Scored under the maxima so far (a segment's first tile has none); where they do not serve this tile, without any, for
        // new ones, and under those.  (One loop around one copy of the scoring, since the code has to come through the
        // instruction cache: three copies took 30.8 instead of 30.2 us for drafted tokens, 57.7 instead of 54.1 for heads of 64.)
        bool under = j > 0, final = false;
#pragma unroll 1
        for (;;) {
          score(under ? row_m : row_zero);
          if (under) {
            if (final) break;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < TPR * CH; i += 2) top = max3(top, y[i], y[i + 1]);
            if (bar_all(bar, kGroup, ok && !(top > kOver))) break;
            under = false;
            continue;
          }
          if (!bar_all(bar, kGroup, ok)) { failed = true; break; }
          // new maxima of the group's rows and what a weight of the old is worth under them: a lane a row
          float x[CH];
#pragma unroll
          for (int i = 0; i < CH; ++i) x[i] = TPR == 1 ? y[i] : fmaxf(y[i], y[(TPR - 1) * CH + i]);
          warp_rows<CH, true>(x, lane);
          const int row = lane / (32 / CH);
          if (lane % (32 / CH) == 0) my_red[(warp & 3) * CH + row] = x[0];
          bar_sync(bar, kGroup);
          const float t = fmaxf(fmaxf(my_red[row], my_red[CH + row]), fmaxf(my_red[2 * CH + row], my_red[3 * CH + row]));
          const float old = row_m[r0 + row], raised = t - old > kNominal ? t - kNominal : old;
          const float fac = raised == old ? 1.0f : fast_exp2(old - raised);
          bar_sync(bar, kGroup);  // everyone has read the old maxima
          if ((warp & 3) == 0 && lane % (32 / CH) == 0) {
            row_m[r0 + row] = raised;
            row_fac[r0 + row] = fac;
          }
          bar_sync(bar, kGroup);
          if (j > 0) {
            ok = wait_pv(gt - 1) && ok;
            tc_fence_after();
          }
#pragma unroll
          for (int c = 0; c < CH; c += 8) {
            float2 f[4];
            load_row<8>(row_fac + r0 + c, f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              l[c + 2 * i] *= f[i].x;
              l[c + 2 * i + 1] *= f[i].y;
            }
            if (j > 0) scale_cols8<3>(lanes + kColO + c, R, f);
          }
          tmem_st_wait();
          under = final = true;
        }
        if (failed) break;
#pragma unroll
        for (int e = 0; e < TPR; ++e) {
          float* const z = y + e * CH;
#pragma unroll
          for (int i = 0; i < CH; i += 2) {
            z[i] = fast_exp2(z[i]);
            z[i + 1] = fast_exp2(z[i + 1]);
            const float2 v = fma2(make_float2(z[i], z[i + 1]), both(inv), make_float2(l[i], l[i + 1]));
            l[i] = v.x;
            l[i + 1] = v.y;
          }
          // MN-major without swizzle: 16 columns of a token, the next rows' tokens; then the next 16 columns
          uint8_t* const at = gbase + Y::kOffP + buf * Y::kP + e * (kRows * PC) + tid * 16;
          if constexpr (CH < 16) {
            uint32_t h[2], m[2], l3[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) split3<true>(z + 4 * i, h[i], m[i], l3[i]);
            *reinterpret_cast<uint4*>(at) = make_uint4(h[0], h[1], m[0], m[1]);
            *reinterpret_cast<uint2*>(at + 16 * kRows) = make_uint2(l3[0], l3[1]);
          } else {
#pragma unroll
            for (int c = 0; c < CH; c += 16) {
              uint32_t t[3][4];
#pragma unroll
              for (int i = 0; i < 4; ++i) split3<true>(z + c + 4 * i, t[0][i], t[1][i], t[2][i]);
#pragma unroll
              for (int k = 0; k < 3; ++k)
                *reinterpret_cast<uint4*>(at + ((r0 + c) / 16 + k * (R / 16)) * (16 * kRows)) =
                    make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]);
            }
          }
        }
        tc_fence_before();
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_local(p_full0 + 8u * buf);
      }
      ring += 2 * w.n;
      const bool whole = w.n == w.all;
      float* const part = p.parts + (2 * static_cast<int64_t>(blockIdx.x) + (w.begin >= first ? 1 : 0)) * Y::kPartFloats;
      if (active && !failed) {
        warp_rows<CH, false>(l, lane);  // the rows' sums
        if (lane % (32 / CH) == 0) my_red[(warp & 3) * CH + lane / (32 / CH)] = l[0];
        bar_sync(bar, kGroup);
        if (tid < CH && r0 + tid < rows) {
          const float sum = (my_red[tid] + my_red[CH + tid]) + (my_red[2 * CH + tid] + my_red[3 * CH + tid]);
          const float m = row_m[r0 + tid];
          if (!whole) {
            part[r0 + tid] = m;
            part[R + r0 + tid] = sum;
          } else if (p.a.lse) {
            const int row = w.sq * R + r0 + tid;
            const int32_t tk = g.token_of(row);
            p.a.lse[static_cast<int64_t>(w.r0 + tk) * p.a.nh + w.sh * g.group + row - tk * g.group] =
                sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
          }
          row_fac[r0 + tid] = sum == 0.0f ? 0.0f : 1.0f / sum;
        }
        bar_sync(bar, kGroup);
        ok = wait_pv(gt - 1) && ok;
        tc_fence_after();
        constexpr int kCols = CH < 16 ? 8 : 16;
        const int dl = HD == 128 ? tid : (warp & 3) * 16 + lane;  // the thread's column of the head (64: lanes 0 .. 15)
#pragma unroll
        for (int c = 0; c < CH; c += kCols) {
          float2 o[kCols / 2];
          load_sums<R, kCols>(lanes + kColO + c, o);
          if (!ok || (HD == 64 && lane >= 16)) continue;
#pragma unroll
          for (int i = 0; i < kCols; ++i) {
            const int r = r0 + c + i;
            const float v = i & 1 ? o[i / 2].y : o[i / 2].x;
            if (r >= rows) break;
            if (whole) {
              const float f = row_fac[r];
              const __nv_bfloat16 out = __float2bfloat16_rn(f == 0.0f ? 0.0f : v * f);
              p.a.o[row_at[r] + dl] = *reinterpret_cast<const uint16_t*>(&out);
            } else {
              part[2 * R + r * HD + dl] = v;
            }
          }
        }
        tc_fence_before();
      }
      ok = ok && !failed;
      if (whole) continue;
      // the last of the row tile's runs joins their parts
      if (!bar_all(bar_every, kSoft, ok)) { ok = false; break; }
      const int32_t c0 = static_cast<int32_t>(w.begin / run), c1 = static_cast<int32_t>((w.begin + w.all - 1) / run);
      if (threadIdx.x == 0) {
        const uint32_t last = static_cast<uint32_t>(c1 - c0);
        uint32_t old;  // releases what the barrier's threads wrote, acquires what the runs before did
        asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(old) : "l"(p.counters + c0), "r"(last) : "memory");
        *merge_flag = old == last;
      }
      bar_sync(bar_every, kSoft);
      if (*merge_flag) {
        auto part_of = [&](int32_t c) { return p.parts + (2 * static_cast<int64_t>(c) + (c == c0 ? 1 : 0)) * Y::kPartFloats; };
        // the rows' maxima and sums over all parts: the threads of a row share them
        constexpr int kPer = kSoft / R;  // 4 to 16
        const int mr = threadIdx.x / kPer, mi = threadIdx.x % kPer;
        float m = kNoMax, sum = 0.0f;
        for (int32_t c = c0 + mi; c <= c1; c += kPer) {
          const float pm = __ldcg(part_of(c) + mr), pl = __ldcg(part_of(c) + R + mr);
          if (mr < rows) {
            const float top = fmaxf(m, pm);
            sum = sum * fast_exp2(m - top) + pl * fast_exp2(pm - top);
            m = top;
          }
        }
#pragma unroll
        for (int o = 1; o < kPer; o <<= 1) {
          const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, sum, o);
          const float top = fmaxf(m, om);
          // (written alike in both lanes: they get the same bits)
          const float mine = sum * fast_exp2(m - top), other = os * fast_exp2(om - top);
          sum = (mi & o) ? other + mine : mine + other;
          m = top;
        }
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (p.a.lse && mi == 0 && mr < rows) {
          const int row = w.sq * R + mr;
          const int32_t tk = g.token_of(row);
          p.a.lse[static_cast<int64_t>(w.r0 + tk) * p.a.nh + w.sh * g.group + row - tk * g.group] =
              sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
        }
        // the parts' weights, 128 parts at a time, over the weights' buffers (no product is under way), then the
        // accumulators: kItems vectors of four columns a thread, kAt of them at a time (few rows have many parts, many
        // rows few), 16 loads at once
        float* const weight = reinterpret_cast<float*>(gbase + Y::kOffP);  // [R][128]
        constexpr int kItems = R * HD / 4 / kSoft, kAt = R == 8 ? 1 : kItems > 4 ? 4 : kItems, kDeep = 16 / kAt;
        float acc[kItems][4] = {};
        for (int32_t cb = c0; cb <= c1; cb += 128) {
          const int32_t count = min(128, c1 + 1 - cb);
          for (int32_t c = mi; c < count; c += kPer)
            weight[mr * 128 + c] = mr < rows ? fast_exp2(__ldcg(part_of(cb + c) + mr) - m) * by : 0.0f;
          bar_sync(bar_every, kSoft);
#pragma unroll
          for (int e0 = 0; e0 < kItems; e0 += kAt) {
            if ((e0 * kSoft + static_cast<int>(threadIdx.x)) / (HD / 4) >= rows) break;
            for (int32_t c = 0; c < count; c += kDeep) {
              float4 v[kDeep][kAt];
#pragma unroll
              for (int k = 0; k < kDeep; ++k)
#pragma unroll
                for (int e = 0; e < kAt; ++e) {
                  const int at = (e0 + e) * kSoft + threadIdx.x;
                  v[k][e] = make_float4(0.f, 0.f, 0.f, 0.f);
                  if (c + k < count && at / (HD / 4) < rows)
                    v[k][e] = __ldcg(reinterpret_cast<const float4*>(part_of(cb + c + k) + 2 * R) + at);
                }
#pragma unroll
              for (int k = 0; k < kDeep; ++k)
#pragma unroll
                for (int e = 0; e < kAt; ++e) {
                  const int r = ((e0 + e) * kSoft + static_cast<int>(threadIdx.x)) / (HD / 4);
                  const float f = c + k < count ? weight[r * 128 + c + k] : 0.0f;
                  acc[e0 + e][0] = fmaf(v[k][e].x, f, acc[e0 + e][0]);
                  acc[e0 + e][1] = fmaf(v[k][e].y, f, acc[e0 + e][1]);
                  acc[e0 + e][2] = fmaf(v[k][e].z, f, acc[e0 + e][2]);
                  acc[e0 + e][3] = fmaf(v[k][e].w, f, acc[e0 + e][3]);
                }
            }
          }
          bar_sync(bar_every, kSoft);
        }
#pragma unroll
        for (int e = 0; e < kItems; ++e) {
          const int at = e * kSoft + threadIdx.x, r = at / (HD / 4);
          uint2 out;
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(out.x) : "f"(acc[e][1]), "f"(acc[e][0]));
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(out.y) : "f"(acc[e][3]), "f"(acc[e][2]));
          if (r < rows) *reinterpret_cast<uint2*>(p.a.o + row_at[r] + 4 * (at % (HD / 4))) = out;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Y::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc<1>(tmem, Y::kTmem);
  }
}

// ---------------------------------------------------------------- many rows a key/value head
// Row tiles of 128 rows (heads of 128): the rows are the M of both products, a thread pair's each,
//   S [128 rows, 128 tokens] = (Q_hi + Q_lo) K^T,      O [128 rows, 128] += (P_h + P_m + P_l) V,
// with queries and weights in tensor memory and the codes as B operands, K as it lies, V MN-major.  Against the other
// kernel's products, whose operands both come from shared memory (1,300 cycles for a tile of 128 tokens and 64 rows with
// two terms of both), the products of a tile of 128 rows take 1,280.  All terms add into one accumulator, so they have one unit: a
// query is hi + lo with lo = e4m3(x - hi), 4 + 4 significant bits down to lo's least step, 2^-9, exact but for 2^-19 of its row's
// largest element, which lies in (224, 448]; a weight is three e5m2 numbers, within 2^-9 of it from 2^-8 on and within e5m2's half
// step, 2^-17, below: 2^-31 of the row's largest, which is 2^kNominalRows or more.
// Thread (row, quarter c) has the row's tokens 32 c .. 32 c + 31 of a tile.  The four agree on the row's maximum through
// shared memory; raising it is lazy, as there, row by row.
// Two prompts' chunks of 1023 tokens on 6001 and 8191 (32 / 8 heads of 128, 213 GFLOP) take 264 us, 0.8 PFLOP/s, bound by
// the softmax's arithmetic.  The products by themselves, the softmax's threads only keeping pace, take 188: 1,280 cycles a tile
// would be 115, the rest is that a tile's scores, its weights and their product follow one another.  In a form with two terms a
// weight (257 us): two threads a row 284; the accumulators raised before the weights are made, and only those of the rows
// that have to be, 266; rows read and written by their own lanes 261; the other kernel with tiles of 64 rows 386.
constexpr float kNominalRows = 14.0f;
struct KvMany {
  static constexpr int kHd = 128, kR = 128, kTpr = 1, kTok = kRows, kHead = 4, kPages = kTok / 16;
  static constexpr int kShare = 4;  // threads a row
  static constexpr int kSoft = 128 * kShare, kTmaWarp = 4 * kShare, kMmaWarp = kTmaWarp + 1, kThreads = kSoft + 64, kSlots = 12;
  static constexpr uint32_t kTile = kRows * 128, kTmem = 512;
  static constexpr uint32_t kColO = 256, kColQ = 384;  // scores twice, accumulators, queries (32 columns hi, 32 lo)
  static constexpr uint32_t kBarFull = 0, kBarEmpty = 8 * kSlots, kBarScale = 16 * kSlots, kBarRest = kBarScale + 8 * kScaleRing;
  static constexpr uint32_t kOffScale = 640, kOffEx = kOffScale + kScaleRing * 8 * kPages, kOffRing = 7 * 1024;
  static constexpr uint32_t kSmem = kOffRing + kSlots * kTile + 1024;
  static constexpr int kPartFloats = kR * (kHd + 2);
  static_assert(kOffEx + 2 * kShare * 128 * 4 <= kOffRing, "exchange");
};

// D[tmem] (+)= A[tmem] B[smem], A: a row a lane, four e4m3 elements a column.
__device__ __forceinline__ void umma_f8_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], db, %4, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Four values as the words of either term, hi + lo.
__device__ __forceinline__ void split4(const float* x, uint32_t& hi, uint32_t& lo) {
  uint16_t h[2], l[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t h16, back;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h16) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(h[i]) : "r"(h16));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(h[i]));
    const __half2 rest = __hsub2(*reinterpret_cast<const __half2*>(&h16), *reinterpret_cast<const __half2*>(&back));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(l[i]) : "r"(*reinterpret_cast<const uint32_t*>(&rest)));
  }
  hi = h[0] | static_cast<uint32_t>(h[1]) << 16;
  lo = l[0] | static_cast<uint32_t>(l[1]) << 16;
}

// Four lanes' four vectors each, exchanged: vector i of lane c for vector c of lane i.
__device__ __forceinline__ void exchange4(uint4 (&r)[4], int lane) {
  auto swap = [&](uint4& a, uint4& b, int o) {  // the lower lane gives b for the upper one's a
    const bool up = (lane & o) != 0;
    uint4 give = up ? a : b;
    give.x = __shfl_xor_sync(0xffffffffu, give.x, o);
    give.y = __shfl_xor_sync(0xffffffffu, give.y, o);
    give.z = __shfl_xor_sync(0xffffffffu, give.z, o);
    give.w = __shfl_xor_sync(0xffffffffu, give.w, o);
    (up ? a : b) = give;
  };
  swap(r[0], r[1], 1);
  swap(r[2], r[3], 1);
  swap(r[0], r[2], 2);
  swap(r[1], r[3], 2);
}

__global__ void __launch_bounds__(KvMany::kThreads, 1)
    kv_attn_rows_kernel(const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv, const KvTcArgs p) {
  using Y = KvMany;
  constexpr int NS = Y::kSlots, HD = 128, R = Y::kR, kTok = Y::kTok, C = Y::kShare, W = 128 / C;  // W columns a thread
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* const gbase = smem_raw + (base - raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full0 = base + Y::kBarFull, empty0 = base + Y::kBarEmpty, scale_full0 = base + Y::kBarScale,
                 s_full0 = base + Y::kBarRest, p_full0 = s_full0 + 16, pv_done0 = p_full0 + 16, q_full = pv_done0 + 16,
                 final_bar = q_full + 8;
  static_assert(Y::kBarRest + 3 * 16 + 2 * 8 <= 400, "barriers");
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(gbase + 400);
  int32_t* const merge_flag = reinterpret_cast<int32_t*>(gbase + 404);
  int32_t* const start = reinterpret_cast<int32_t*>(gbase + 408);
  int64_t* const scan = reinterpret_cast<int64_t*>(gbase + 424);
  int32_t* const longest = reinterpret_cast<int32_t*>(gbase + 424 + 8 * (Y::kThreads / 32));
  static_assert(424 + 12 * (Y::kThreads / 32) <= Y::kOffScale, "start");
  float* const scales = reinterpret_cast<float*>(gbase + Y::kOffScale);
  float* const ex = reinterpret_cast<float*>(gbase + Y::kOffEx);  // [2][C][128]: what the threads of a row tell each other

  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(full0 + 8u * i, 1);
      mbar_init(empty0 + 8u * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full0 + 8u * i, 1);
      mbar_init(p_full0 + 8u * i, Y::kSoft / 32);
      mbar_init(pv_done0 + 8u * i, 1);
    }
    for (int i = 0; i < kScaleRing; ++i) mbar_init(scale_full0 + 8u * i, 1);
    mbar_init(q_full, Y::kSoft / 32);
    mbar_init(final_bar, 1);
    fence_mbar_init_cluster();
  }
  if (warp == Y::kMmaWarp) tmem_alloc<1>(smem_u32(tmem_slot), Y::kTmem);
  if (warp == Y::kTmaWarp && lane == 0) {
    prefetch_tmap(&tmk);
    prefetch_tmap(&tmv);
  }
  grid_launch_dependents();
  grid_dependency_wait();
  const KvGeom& g = p.g;
  int64_t run, first;
  KvWalk<Y> w = find_run<Y>(p, scan, longest, start, run, first);
  const uint32_t tmem = *tmem_slot;
  const KvCacheDev& kv = p.a.cache;
  bool ok = true;

  if (warp == Y::kTmaWarp) {
    copy_tiles<Y>(tmk, tmv, p, w, base, scales);
  } else if (warp == Y::kMmaWarp) {
    constexpr uint32_t idesc_s = idesc_f8(R, kTok, false, false), idesc_o = idesc_f8(R, HD, false, true, true);
    constexpr uint32_t kHi = desc_hi(1024, 2);
    const bool issuer = elect_one();
    int slot = 0;
    uint32_t ph = 0, gt = 0, seg = 0;
    auto step = [&] {
      if (++slot == NS) { slot = 0; ph ^= 1u; }
    };
    auto issue_s = [&](uint32_t buf) -> bool {
      if (!mbar_wait_warp(full0 + 8u * slot, ph, p.wc)) return false;
      tc_fence_after();
      if (issuer) {
        const uint32_t bd = desc_lo(base + Y::kOffRing + slot * Y::kTile, 16);
#pragma unroll
        for (int k = 0; k < 8; ++k)  // hi, then lo
          umma_f8_ts(tmem + 128 * buf, tmem + Y::kColQ + 8 * k, bd + 2 * (k % 4), kHi, idesc_s, k > 0 ? 1u : 0u);
        umma_commit<1>(s_full0 + 8u * buf);
        umma_commit<1>(empty0 + 8u * slot);
      }
      step();
      return true;
    };
    while (ok && w.next(g)) {
      if (!mbar_wait_warp(q_full, seg & 1, p.wc)) { ok = false; break; }
      tc_fence_after();
      if (!issue_s(gt & 1) || (w.n > 1 && !issue_s((gt + 1) & 1))) { ok = false; break; }
      ++seg;
#pragma unroll 1
      for (int32_t j = 0; j < w.n; ++j, ++gt) {
        const uint32_t buf = gt & 1;
        if (!mbar_wait_warp(full0 + 8u * slot, ph, p.wc) || !mbar_wait_warp(p_full0 + 8u * buf, (gt >> 1) & 1, p.wc)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (issuer) {
          const uint32_t bd = desc_lo(base + Y::kOffRing + slot * Y::kTile, 16);
#pragma unroll
          for (int k = 0; k < 12; ++k)  // 32 tokens at a time, whose words lie over their scores: 8 columns a term
            umma_f8_ts(tmem + Y::kColO, tmem + 128 * buf + 32 * (k % 4) + 8 * (k / 4), bd + 256 * (k % 4), kHi, idesc_o,
                       (j > 0 || k > 0) ? 1u : 0u);
          umma_commit<1>(pv_done0 + 8u * buf);
          umma_commit<1>(empty0 + 8u * slot);
        }
        step();
        if (j + 2 < w.n && !issue_s(buf)) { ok = false; break; }
      }
    }
    if (issuer) umma_commit<1>(final_bar);
    __syncwarp();
    drain(final_bar, 0);  // every MMA has completed before TMEM is released
  } else {
    const int quarter = warp & 3, c = warp >> 2, row = quarter * 32 + lane;
    constexpr int kEvery = 5;
    const int page_shift = 31 - __clz(kv.page);
    // the row's threads meet; their word k, theirs in order
    auto others = [&](int k, float mine, auto join) {
      float v = mine;
#pragma unroll
      for (int i = 1; i < C; ++i) v = join(v, ex[k * (128 * C) + ((c + i) % C) * 128 + row]);
      return v;
    };
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    uint32_t gt = 0, ring = 0;
    // (see the other kernel's)
    auto wait_pv = [&](uint32_t t) { return mbar_wait_warp(pv_done0 + 8u * (t & 1), (t >> 1) & 1, p.wc); };
    // Rows come and go four at a time, 64 bytes of each by the four lanes whose rows they are (by the row's own
    // lane, a line a row and instruction, 8 prompts of 512 took 78 us instead of 74).  Vector i of the
    // lane is part of row i of the four: its offset in rows ld elements apart, -1 behind the last row.
    auto place = [&](const KvWalk<Y>& v, int i, int64_t ld) -> int64_t {
      const int32_t at = v.sq * R + quarter * 32 + (lane & ~3) + i, tk = g.token_of(at);
      return at < v.rows_n * g.group ? (v.r0 + tk) * ld + (v.sh * g.group + at - tk * g.group) * HD + W * c + 8 * (lane & 3) : -1;
    };
    static_assert(W == 32, "four vectors a row");
    auto ask = [&](const KvWalk<Y>& v, uint4 (&q)[W / 8]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t from = place(v, i, p.a.ldq);
        q[i] = make_uint4(0u, 0u, 0u, 0u);
        if (from >= 0) q[i] = *reinterpret_cast<const uint4*>(p.a.q + from);
      }
    };
    while (w.next(g)) {
      if (!bar_all(kEvery, Y::kSoft, ok)) { ok = false; break; }
      const int32_t at = w.sq * R + row, tk = g.token_of(at), head = w.sh * g.group + at - tk * g.group;
      const bool mine = at < w.rows_n * g.group;
      const int32_t lim = mine ? w.len - w.rows_n + tk : -1;
      const int32_t sees_all = w.len - w.rows_n + g.token_of(w.sq * R) + 1;  // (the first row's, the others' at least that)
      float f;
      {
        uint4 q[W / 8];
        ask(w, q);
        exchange4(q, lane);
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < W / 8; ++k) {
          const uint32_t u[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max(top, max(u[e] << 16 & 0x7fffffffu, u[e] & 0x7fff0000u));
        }
        ex[c * 128 + row] = __uint_as_float(top);
        bar_sync(1 + quarter, 32 * C);
        top = __float_as_uint(others(0, __uint_as_float(top), [](float a, float b) {
          return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));  // (as integers: NaN is the largest)
        }));
        // 2^-e brings the largest element into (224, 448]; a row that is not finite has NaN as its factor
        const int e = max(static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), kLeastExp);
        const bool bad = top >= 0x7f800000u;
        const float by = bad ? 0.0f : __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        f = bad ? __uint_as_float(0x7fffffffu) : __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * p.a.scale_log2;
        uint32_t hi[W / 4], lo[W / 4];
#pragma unroll
        for (int k = 0; k < W / 8; ++k) {
          const uint32_t u[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
          float x[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[2 * i] = bad ? 0.0f : __uint_as_float(u[i] << 16) * by;
            x[2 * i + 1] = bad ? 0.0f : __uint_as_float(u[i] & 0xffff0000u) * by;
          }
          split4(x, hi[2 * k], lo[2 * k]);
          split4(x + 4, hi[2 * k + 1], lo[2 * k + 1]);
        }
        tmem_st8(lanes + Y::kColQ + W / 4 * c, hi);
        tmem_st8(lanes + Y::kColQ + 32 + W / 4 * c, lo);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_local(q_full);
      }
      float m = kNoMax, l = 0.0f;
      bool failed = false;
#pragma unroll 1
      for (int32_t j = 0; j < w.n; ++j, ++gt) {
        const uint32_t buf = gt & 1, sbuf = lanes + 128 * buf + W * c;
        const int32_t tile = (w.t0 + j) * kTok;
        ok = mbar_wait_warp(scale_full0 + 8u * (gt % kScaleRing), (gt / kScaleRing) & 1, p.wc) && ok;
        const float* const sc = scales + (gt % kScaleRing) * (2 * Y::kPages);
        float ks[W / 16], lsv[W / 16], inv[W / 16];  // of 16 tokens each (see the other kernel)
#pragma unroll
        for (int i = 0; i < W / 16; ++i) {
          const int at_page = (W * c + 16 * i) >> page_shift;
          ks[i] = sc[at_page];
          uint32_t vb = __float_as_uint(sc[Y::kPages + at_page]);
          if (vb == 0u) vb = kLeastScale;
          if (vb >= 0x7f800000u) {
            ks[i] = __uint_as_float(0x7fffffffu);
            vb = 127u << 23;
          }
          lsv[i] = static_cast<float>(static_cast<int>(vb >> 23) - 127);
          inv[i] = __uint_as_float((254u - (vb >> 23)) << 23);
        }
        ok = mbar_wait_warp(s_full0 + 8u * buf, (gt >> 1) & 1, p.wc) && ok;
        tc_fence_after();
        if (c == 0 && tile + kTok > w.vis) {
          // the values behind the last visible token become zeros
          const uint32_t vat = ring + min(2, w.n) + j + max(0, min(j, w.n - 2)), sl = vat % NS;
          ok = mbar_wait_warp(full0 + 8u * sl, (vat / NS) & 1, p.wc) && ok;
          uint4* const v = reinterpret_cast<uint4*>(gbase + Y::kOffRing + sl * Y::kTile);
#pragma unroll 1
          for (int32_t i = max(w.vis - tile, 0) * 8 + row; i < kRows * 8; i += 128) v[i] = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async_smem();
        }
        uint32_t v[32];
        static_assert(W == 32, "one load");
        tmem_ld32(sbuf, v);
        tmem_ld_wait();
        float x[W], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < W; i += 2) {
          const float2 t = fma2(make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])),
                                both(f * ks[i / 16]), both(lsv[i / 16]));
          x[i] = t.x;
          x[i + 1] = t.y;
        }
        if (tile + kTok > sees_all) {
          const int32_t sees = lim - tile - W * c;  // the thread's last visible token
#pragma unroll
          for (int i = 0; i < W; ++i)
            if (i > sees) x[i] = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < W; i += 2) top = max3(top, x[i], x[i + 1]);
        ex[buf * (128 * C) + c * 128 + row] = top;
        if (!bar_all(1 + quarter, 32 * C, ok)) { failed = true; break; }
        top = others(buf, top, [](float a, float b) { return fmaxf(a, b); });
        // Where some row has to be raised, those that only could be are too: the accumulators' turn costs the same.
        const bool any = __any_sync(0xffffffffu, top - m > kOver);
        float fac = 1.0f;
        if (any) {
          const float to = top - m > kNominalRows ? top - kNominalRows : m;
          fac = to == m ? 1.0f : fast_exp2(m - to);
          m = to;
          l *= fac;
        }
        uint32_t t[3][W / 4];
#pragma unroll
        for (int i = 0; i < W; i += 16) {
          float2 sum = both(0.0f);
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float2 y = fma2(both(m), both(-1.0f), make_float2(x[i + e], x[i + e + 1]));
            x[i + e] = fast_exp2(y.x);
            x[i + e + 1] = fast_exp2(y.y);
            sum = fma2(make_float2(x[i + e], x[i + e + 1]), both(1.0f), sum);
          }
          l = fmaf(sum.x + sum.y, inv[i / 16], l);
#pragma unroll
          for (int e = 0; e < 4; ++e) split3<false>(x + i + 4 * e, t[0][i / 4 + e], t[1][i / 4 + e], t[2][i / 4 + e]);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) tmem_st8(sbuf + 8 * k, t[k]);
        if (any && j > 0) {  // (by now the product before has mostly completed)
          ok = wait_pv(gt - 1) && ok;
          tc_fence_after();
          const float2 f4[4] = {both(fac), both(fac), both(fac), both(fac)};
#pragma unroll 1
          for (int i = 0; i < W; i += 8) scale_cols8<1>(lanes + Y::kColO + W * c + i, 0, f4);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_local(p_full0 + 8u * buf);
      }
      ring += 2 * w.n;
      const bool whole = w.n == w.all;
      float* const part = p.parts + (2 * static_cast<int64_t>(blockIdx.x) + (w.begin >= first ? 1 : 0)) * Y::kPartFloats;
      uint16_t* const out = p.a.o + (w.r0 + tk) * p.a.ldo + head * HD + W * c;
      const int64_t lse_at = static_cast<int64_t>(w.r0 + tk) * p.a.nh + head;
      if (!failed) {
        // (the exchange of the tile before last is free: the row's threads have met since)
        float* const sums = ex + (gt & 1) * (128 * C) + row;
        sums[c * 128] = l;
        bar_sync(1 + quarter, 32 * C);
        float sum = sums[0];  // in one order: the same bits in every thread
#pragma unroll
        for (int i = 1; i < C; ++i) sum += sums[i * 128];
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (mine && c == 0) {
          if (!whole) {
            part[row] = m;
            part[R + row] = sum;
          } else if (p.a.lse) {
            p.a.lse[lse_at] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
          }
        }
        ok = wait_pv(gt - 1) && ok;
        tc_fence_after();
        if (whole) {
          uint4 two[W / 8];
#pragma unroll
          for (int i = 0; i < W; i += 16) {
            uint32_t o[16], u[8];
            tmem_ld16(lanes + Y::kColO + W * c + i, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float a = by == 0.0f ? 0.0f : __uint_as_float(o[2 * e]) * by;
              const float b = by == 0.0f ? 0.0f : __uint_as_float(o[2 * e + 1]) * by;
              asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[e]) : "f"(b), "f"(a));
            }
            two[i / 8] = make_uint4(u[0], u[1], u[2], u[3]);
            two[i / 8 + 1] = make_uint4(u[4], u[5], u[6], u[7]);
          }
          exchange4(two, lane);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t to = place(w, i, p.a.ldo);
            if (ok && to >= 0) *reinterpret_cast<uint4*>(p.a.o + to) = two[i];
          }
        } else {
#pragma unroll 1
          for (int i = 0; i < W; i += 16) {
            uint32_t o[16];
            tmem_ld16(lanes + Y::kColO + W * c + i, o);
            tmem_ld_wait();
            if (!mine || !ok) continue;
            uint4* const to = reinterpret_cast<uint4*>(part + 2 * R + row * HD + W * c + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) to[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
        tc_fence_before();
      }
      ok = ok && !failed;
      if (whole) continue;
      // the last of the row tile's runs joins their parts, a thread its quarter of its row
      if (!bar_all(kEvery, Y::kSoft, ok)) { ok = false; break; }
      const int32_t c0 = static_cast<int32_t>(w.begin / run), c1 = static_cast<int32_t>((w.begin + w.all - 1) / run);
      if (threadIdx.x == 0) {
        const uint32_t last = static_cast<uint32_t>(c1 - c0);
        uint32_t old;
        asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(old) : "l"(p.counters + c0), "r"(last) : "memory");
        *merge_flag = old == last;
      }
      bar_sync(kEvery, Y::kSoft);
      if (*merge_flag && mine) {
        float top = kNoMax, sum = 0.0f, acc[W];
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] = 0.0f;
#pragma unroll 1
        for (int32_t r = c0; r <= c1; ++r) {
          const float* const q = p.parts + (2 * static_cast<int64_t>(r) + (r == c0 ? 1 : 0)) * Y::kPartFloats;
          float4 v[W / 4];
#pragma unroll
          for (int i = 0; i < W / 4; ++i) v[i] = __ldcg(reinterpret_cast<const float4*>(q + 2 * R + row * HD + W * c) + i);
          const float pm = __ldcg(q + row), pl = __ldcg(q + R + row), to = fmaxf(top, pm);
          const float fa = fast_exp2(top - to), fb = fast_exp2(pm - to);
          sum = sum * fa + pl * fb;
          top = to;
#pragma unroll
          for (int i = 0; i < W / 4; ++i) {
            acc[4 * i] = acc[4 * i] * fa + v[i].x * fb;
            acc[4 * i + 1] = acc[4 * i + 1] * fa + v[i].y * fb;
            acc[4 * i + 2] = acc[4 * i + 2] * fa + v[i].z * fb;
            acc[4 * i + 3] = acc[4 * i + 3] * fa + v[i].w * fb;
          }
        }
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (p.a.lse && c == 0) p.a.lse[lse_at] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
#pragma unroll
        for (int i = 0; i < W; i += 8) {
          uint32_t two[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;"
                : "=r"(two[e])
                : "f"(by == 0.0f ? 0.0f : acc[i + 2 * e + 1] * by), "f"(by == 0.0f ? 0.0f : acc[i + 2 * e] * by));
          *reinterpret_cast<uint4*>(out + i) = make_uint4(two[0], two[1], two[2], two[3]);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Y::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc<1>(tmem, Y::kTmem);
  }
}

PFN_cuTensorMapEncodeTiled_v12000 g_enc = nullptr;
std::once_flag g_enc_once;

// Codes as rows of 128 bytes (a token of 128 elements, or two of 64), boxes of one page and head.
bool tmap_codes(CUtensorMap* m, const void* ptr, int32_t d, int64_t rows, int32_t page) {
  std::call_once(g_enc_once, [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q{};
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      g_enc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  });
  if (!g_enc) return false;
  const cuuint64_t dims[2] = {128, static_cast<cuuint64_t>(rows * d / 128)};
  const cuuint64_t strides[1] = {128};
  const cuuint32_t box[2] = {128, static_cast<cuuint32_t>(page * d / 128)};
  const cuuint32_t estr[2] = {1, 1};
  return g_enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count() {
  int sm = 152, dev = 0;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev);
  return sm;
}

constexpr size_t kCounterBytes = 4096;  // up to 1024 CTAs

template <class Y>
cudaError_t run_kv(void (*kern)(CUtensorMap, CUtensorMap, KvTcArgs), int ctas, const KvAttnArgs& a, cudaStream_t st) {
  constexpr int HD = Y::kHd;
  CUtensorMap tk, tv;
  const int64_t rows = static_cast<int64_t>(a.cache.n_pages) * a.cache.nkv * a.cache.page;
  if (!tmap_codes(&tk, a.cache.k_codes, HD, rows, a.cache.page) || !tmap_codes(&tv, a.cache.v_codes, HD, rows, a.cache.page))
    return cudaErrorInvalidValue;
  KvTcArgs p{};
  p.a = a;
  if (!launch_wait_ctl(&p.wc)) return cudaErrorInvalidDevice;
  p.a.status = p.wc.status_word;
  p.g = KvGeom{a.row_start, a.seq_len, a.B, a.nh / a.cache.nkv, a.cache.nkv,
               static_cast<uint32_t>(((uint64_t(1) << 32) + a.nh / a.cache.nkv - 1) / (a.nh / a.cache.nkv)), a.T,
               static_cast<int64_t>(a.cache.max_pages) * a.cache.page};
  p.counters = static_cast<uint32_t*>(a.workspace);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + kCounterBytes);
  static std::atomic<uint64_t> ready{0};  // devices on which the kernel may use its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Y::kSmem);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(std::min(ctas * sm_count(), 1024)));
  cfg.blockDim = dim3(Y::kThreads);
  cfg.dynamicSmemBytes = Y::kSmem;
  cfg.stream = st;
  // the kernel waits by itself for the launch ahead; its first steps run beside that one's end
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, tk, tv, p);
}

// Rows of a tile: by what an average sequence has a key/value head (any number is right).  16 sequences of 4096 tokens, 8
// key/value heads, us with tiles of 8 / 16 / 32 / 128 rows: heads of 128, 4 rows 29.4 / 28.8 / 31.7 / 49.4, 12 rows 33.9 /
// 29.4 / 33.4 / 50, 24 rows 44.8 / 36.8 / 35.2 / 52, 64 rows 117 / 68 / 51 / 56, 96 rows 144 / 104 / 71 / 61, 128 rows 191 / 125 / 90 /
// 66; heads of 64, 4 rows 17.5 / 18.7 / 23.9, 16 rows 24.6 / 19.5 / 24.9, 32 rows 38 / 29 / 28, 128 rows 122 / 84 / 79.  The mean is a
// poor guide to a batch of single tokens with a prompt among them: 128 single tokens on 2048 and a prompt of 512 (32 / 8 heads
// of 128) take 155 us in one call, 129 in two; 32 on 4096 and a prompt of 2048 171 and 146.
template <int HD, int R>
cudaError_t run_few(const KvAttnArgs& a, cudaStream_t st) {
  return run_kv<KvLay<HD, R>>(kv_attn_kernel<HD, R>, KvLay<HD, R>::kCtas, a, st);
}
template <int HD>
cudaError_t run_kv_rows(const KvAttnArgs& a, cudaStream_t st) {
  const int64_t rows = (a.T + a.B - 1) / a.B * (a.nh / a.cache.nkv);
  if (rows <= 8) return run_few<HD, 8>(a, st);
  if (rows <= 16) return run_few<HD, 16>(a, st);
  if (rows <= 64 || HD == 64) return run_few<HD, 32>(a, st);
  return run_kv<KvMany>(kv_attn_rows_kernel, 1, a, st);
}

}  // namespace

size_t kv_attention_ws_bytes(int32_t, int32_t, int32_t d) {
  // two parts for each CTA: two CTAs an SM with tiles of up to 32 rows, one of 128 (heads of 64: of 32)
  const size_t parts = static_cast<size_t>(sm_count()) * 2 * (d == 128 ? 128 : 64) * (static_cast<size_t>(d) + 2) * sizeof(float);
  return (kCounterBytes + parts + 255) / 256 * 256;
}

cudaError_t launch_kv_attention(KvAttnArgs a, cudaStream_t st) {
  return a.cache.d == 128 ? run_kv_rows<128>(a, st) : run_kv_rows<64>(a, st);
}

}  // namespace catq
