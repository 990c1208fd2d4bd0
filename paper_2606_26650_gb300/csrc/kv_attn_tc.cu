// kv_attn_tc.cu — grouped-query attention of new tokens over the paged cache of 8-bit codes, on the tcgen05
// tensor cores with the codes as they lie in the cache: no element of the cache passes through a register.
//
// With few query rows a key/value head, the cached tokens are the long side: they are the M of both products, the
// rows (new token, query head of the group), R of them a CTA's tile, the N:
//   S^T [128 tokens, 2 R] = K [128, d] Q^T,      O^T [d, 2 R] += V^T [d, 128] P^T [128, 2 R].
// A operands are the code tiles that TMA brings page by page (K K-major, V MN-major: the tensor core transposes it), e4m3
// like the cache.  B operands are e4m3 too, as two terms in columns of their own: x = hi + lo / 16 with hi = e4m3(x), lo =
// e4m3(16 (x - hi)), 4 + 4 significant bits.  A bf16 query (8 bits), scaled by a power of two so that its row's largest
// element lies in (224, 448], is exact but for what is 2^-22 of that element; a weight of the values is off by a relative
// 2^-8 at most, as a bf16 weight would be.  (Converting the codes to 16 bits instead would cost the CTAs some 4
// instructions a pair of elements, at 23 elements a cycle and SM more than the loads themselves.)
//
// Scores in base 2: x = (S_hi + S_lo / 16) s_k f + log2 s_v for a token of a page with scales s_k, s_v (powers of two) and
// a row whose query's scale and log2(e) / sqrt(d) are in f; weights of the value codes are w = 2^(x - m), the row's sum adds
// w / s_v, and at the end O = O^T / sum, lse = (m + log2 sum) ln 2, both exact for whichever m was used.  m is the row's
// largest x less 5, so that most weights lie well inside e4m3's range (2^-9 .. 448; hi + lo / 16 resolves 2^-14, 2^-19 of
// the largest), and is raised lazily: only when some x - m passes 8.75 (weights stay below 448) does the CTA agree on new
// maxima and rescale its sums and accumulators.
//
// A CTA has 4 softmax warps (thread t owns token t of a tile: TMEM lane t), a TMA warp and an MMA warp; two CTAs an SM up
// to 32 rows.  Work: the tiles of 128 tokens of all (sequence, key/value head, row tile), in this order as one line, cut
// into equal runs, one a CTA, whatever the sequences' lengths are; they are read on the device, so a captured launch
// follows them.  A run that holds only a part of a row tile's tokens leaves its maxima, sums and accumulators in the
// workspace; the last run of the row tile to finish (a counter, which it leaves at zero) joins them in their order, so
// the result does not depend on which one that is.
//
// Tokens behind a row's own position weigh 0 whatever their scales are; the values behind the last visible token of a tile
// are zeroed in shared memory (what an unfinished page holds there may be anything, NaN codes too).
#include <cuda.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <mutex>

#include "launch.h"
#include "ptx_sm100.cuh"

namespace catq {
namespace {

constexpr int kTok = 128;                    // cached tokens per tile (MMA M of S^T, contraction of O^T)
constexpr int kSoft = 128;                   // softmax threads
constexpr int kTmaWarp = 4, kMmaWarp = 5;
constexpr int kThreads = 6 * 32;
constexpr float kNominal = 5.0f;             // log2 of a weight at the maximum taken
constexpr float kOver = 8.75f;               // raise the maximum past this (2^8.75 < 448)
constexpr float kNoMax = -3e38f;             // maximum of a row that has seen nothing
constexpr float kLoUnit = 0.0625f;           // a lo term's unit

template <int HD, int R>
struct KvLay {
  static constexpr int kCols = 2 * R;                                // N of both products
  static constexpr int kChunk = R < 16 ? R : 16;                     // rows handled at a time
  static constexpr int kCtas = R <= 32 ? 2 : 1;                      // CTAs an SM
  static constexpr uint32_t kTile = kTok * HD;                       // a tile of codes
  static constexpr uint32_t kQ = kCols * HD, kP = kTok * kCols;
  static constexpr uint32_t kRowBytes = R * 4;
  // barriers, tensor-memory address, start of the run | per row: query factor, maximum, last position, sums by warp |
  // Q, P twice, ring
  static constexpr uint32_t kOffF = 512, kOffM = kOffF + kRowBytes, kOffLim = kOffM + kRowBytes,
                            kOffRed = kOffLim + kRowBytes, kOffQ = (kOffRed + 4 * kRowBytes + 127) / 128 * 128,
                            kOffP = kOffQ + kQ, kOffRing = (kOffP + 2 * kP + 1023) / 1024 * 1024;
  static constexpr uint32_t kBudget = kCtas == 2 ? 112 * 1024 : 224 * 1024;
  static constexpr int kSlots0 = (kBudget - 1024 - kOffRing) / kTile;
  static constexpr int kSlots = kSlots0 > 12 ? 12 : kSlots0;
  static constexpr uint32_t kSmem = kOffRing + kSlots * kTile + 1024;
  static constexpr uint32_t kTmem = 3 * kCols <= 64 ? 64 : 3 * kCols <= 128 ? 128 : 3 * kCols <= 256 ? 256 : 512;
  static constexpr int kPartFloats = R * (HD + 2);                   // maxima, sums, accumulators of a part
};

// ---------------------------------------------------------------- the line of tiles
// One sequence's share of the line: `per_head` tiles for each key/value head.
struct KvSeq {
  int32_t r0, n, len;  // first row, rows, cached tokens
  int64_t per_head;
};

struct KvGeom {
  const int32_t *row_start, *seq_len;
  int32_t B, group, nkv;
  int64_t T, max_len;
};

// Tokens that the row tile `q` of a sequence can see.
template <int R>
__device__ __forceinline__ int32_t visible(const KvGeom& g, const KvSeq& s, int32_t q) {
  const int64_t last = min(static_cast<int64_t>(q + 1) * R, static_cast<int64_t>(s.n) * g.group) - 1;
  return max(s.len - s.n + static_cast<int32_t>(last / g.group) + 1, 0);
}
template <int R>
__device__ __forceinline__ int32_t row_tiles(const KvGeom& g, const KvSeq& s) {
  return static_cast<int32_t>((static_cast<int64_t>(s.n) * g.group + R - 1) / R);
}
// A row tile that sees nothing still has a tile: its rows are written.
__device__ __forceinline__ int32_t tiles_of(int32_t vis) { return max((vis + kTok - 1) / kTok, 1); }

template <int R>
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
  const int32_t nq = row_tiles<R>(g, s);
  for (int32_t q = 0; q < nq; ++q) s.per_head += tiles_of(visible<R>(g, s, q));
  return s;
}

// Walks a run's segments: a segment is the run's part of one row tile.
template <int R>
struct KvWalk {
  int64_t at, end;       // line positions still to do
  int32_t b, h, q, t;    // the next tile: sequence, head, row tile, tile of the row tile
  KvSeq s;
  // the segment
  int32_t n;             // its tiles
  int32_t t0;            // first of them
  int32_t all, vis;      // the row tile's tiles and visible tokens
  int64_t begin;         // line position of the row tile's first tile
  int32_t sb, sh, sq;    // its sequence, head, row tile
  KvSeq ss;
  __device__ __forceinline__ bool next(const KvGeom& g) {
    if (at >= end) return false;
    if (s.per_head == 0 || h == g.nkv) {
      do {
        ++b;
        s = load_seq<R>(g, b, nullptr);
      } while (s.per_head == 0);
      h = q = t = 0;
    }
    sb = b; sh = h; sq = q; ss = s;
    vis = visible<R>(g, s, q);
    all = tiles_of(vis);
    t0 = t;
    n = static_cast<int32_t>(min(static_cast<int64_t>(all - t), end - at));
    begin = at - t;
    at += n;
    t = 0;
    if (++q == row_tiles<R>(g, s)) {
      q = 0;
      ++h;
    }
    return true;
  }
};

// ---------------------------------------------------------------- operands
__device__ __forceinline__ float fast_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
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

// Instruction descriptor of kind::f8f6f4: e4m3 A and B, fp32 D.
__host__ __device__ constexpr uint32_t idesc_e4m3(uint32_t M, uint32_t N, bool a_mn, bool b_mn) {
  return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The hi and lo columns of chunk c (rows c kChunk ..) at `base`: 16 columns of both for 8 rows, else 16 and 16.
template <int R>
__device__ __forceinline__ void load_chunk(uint32_t base, int c, uint32_t (&v)[R < 16 ? 16 : 32]) {
  if constexpr (R < 16) {
    tmem_ld16(base, v);
  } else {
    uint32_t(&hi)[16] = *reinterpret_cast<uint32_t(*)[16]>(&v[0]);
    uint32_t(&lo)[16] = *reinterpret_cast<uint32_t(*)[16]>(&v[16]);
    tmem_ld16(base + 16u * c, hi);
    tmem_ld16(base + R + 16u * c, lo);
  }
  tmem_ld_wait();
}
template <int R>
__device__ __forceinline__ void store_chunk(uint32_t base, int c, const uint32_t (&v)[R < 16 ? 16 : 32]) {
  if constexpr (R < 16) {
    tmem_st16(base, v);
  } else {
    tmem_st16(base + 16u * c, *reinterpret_cast<const uint32_t(*)[16]>(&v[0]));
    tmem_st16(base + R + 16u * c, *reinterpret_cast<const uint32_t(*)[16]>(&v[16]));
  }
}

__device__ __forceinline__ void soft_sync() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }

// Sums over a warp of v[0 .. R): afterwards lane l holds those of rows l R / 32 .. in v[0 .. R / 32), or, where R < 32,
// that of row l / (32 / R) in v[0].
template <int R>
__device__ __forceinline__ void warp_row_sums(float (&v)[R], int lane) {
  int n = R;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (n > 1) {
      n /= 2;
      const bool up = (lane & o) != 0;
#pragma unroll
      for (int i = 0; i < R / 2; ++i)
        if (i < n) {
          const float send = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
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
  int32_t min_run;     // least tiles of a run
  WaitCtl wc;
};

template <int HD, int R>
__global__ void __launch_bounds__(kThreads, KvLay<HD, R>::kCtas)
    kv_attn_kernel(const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv, const KvTcArgs p) {
  using Y = KvLay<HD, R>;
  constexpr int NC = Y::kCols, CH = Y::kChunk, NS = Y::kSlots;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* const gbase = smem_raw + (base - raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full0 = base, empty0 = base + 8u * NS, s_full0 = base + 16u * NS, p_full0 = s_full0 + 16,
                 pv_done0 = p_full0 + 16, q_full = pv_done0 + 16, final_bar = q_full + 8;
  static_assert(16 * NS + 3 * 16 + 2 * 8 <= 272, "barriers");
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(gbase + 272);
  int32_t* const merge_flag = reinterpret_cast<int32_t*>(gbase + 276);
  int64_t* const scan = reinterpret_cast<int64_t*>(gbase + 280);             // warps' sums [6]
  int32_t* const start = reinterpret_cast<int32_t*>(gbase + 336);           // b, h, q, t of the run's first tile
  float* const row_f = reinterpret_cast<float*>(gbase + Y::kOffF);
  float* const row_m = reinterpret_cast<float*>(gbase + Y::kOffM);
  int32_t* const row_lim = reinterpret_cast<int32_t*>(gbase + Y::kOffLim);
  float* const red = reinterpret_cast<float*>(gbase + Y::kOffRed);           // [4][R]

  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(full0 + 8u * i, 1);
      mbar_init(empty0 + 8u * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full0 + 8u * i, 1);
      mbar_init(p_full0 + 8u * i, 4);
      mbar_init(pv_done0 + 8u * i, 1);
    }
    mbar_init(q_full, 4);
    mbar_init(final_bar, 1);
    fence_mbar_init_cluster();
  }
  if (warp == kMmaWarp) tmem_alloc<1>(smem_u32(tmem_slot), Y::kTmem);

  // The run of this CTA: every CTA adds up all sequences' tiles, a thread a stretch of them.
  const KvGeom& g = p.g;
  int64_t run, total, first;
  {
    const int32_t per = (g.B + kThreads - 1) / kThreads;
    const int32_t b0 = min(static_cast<int32_t>(threadIdx.x) * per, g.B), b1 = min(b0 + per, g.B);
    int64_t mine = 0;
    for (int32_t b = b0; b < b1; ++b)
      mine += load_seq<R>(g, b, blockIdx.x == 0 ? p.a.status : nullptr).per_head * g.nkv;
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) upto += scan[w];
      total += scan[w];
    }
    run = max((total + gridDim.x - 1) / gridDim.x, static_cast<int64_t>(p.min_run));
    first = run * blockIdx.x;
    if (upto - mine <= first && first < upto) {  // the thread whose stretch holds the run's first tile
      int64_t rest = first - (upto - mine);
      int32_t b = b0;
      KvSeq s = load_seq<R>(g, b, nullptr);
      while (rest >= s.per_head * g.nkv) {
        rest -= s.per_head * g.nkv;
        s = load_seq<R>(g, ++b, nullptr);
      }
      const int32_t h = static_cast<int32_t>(rest / s.per_head);
      rest -= h * s.per_head;
      int32_t q = 0;
      for (int32_t n; rest >= (n = tiles_of(visible<R>(g, s, q))); ++q) rest -= n;
      start[0] = b;
      start[1] = h;
      start[2] = q;
      start[3] = static_cast<int32_t>(rest);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t kColO = 2 * NC;
  KvWalk<R> w;
  w.at = first;
  w.end = min(first + run, total);
  if (w.at < w.end) {
    w.b = start[0];
    w.h = start[1];
    w.q = start[2];
    w.t = start[3];
    w.s = load_seq<R>(g, w.b, nullptr);
  }
  const KvCacheDev& kv = p.a.cache;
  const int32_t ppt = kTok / kv.page;  // pages a tile
  bool ok = true;

  if (warp == kTmaWarp) {
    if (lane == 0) {
      prefetch_tmap(&tmk);
      prefetch_tmap(&tmv);
    }
    int slot = 0, loads = 0;
    uint32_t ph = 1;
    // tile j of the segment into the next slot, a lane a page
    auto load = [&](const CUtensorMap* map, int32_t j) -> bool {
      const int32_t tok = (w.t0 + j) * kTok;
      const int32_t pages = min(max((w.vis - tok + kv.page - 1) / kv.page, 0), ppt);
      int32_t row = 0;
      if (lane < pages) {
        const int32_t id = __ldg(kv.table + static_cast<int64_t>(w.sb) * kv.max_pages + tok / kv.page + lane);
        const bool in = id >= 0 && id < kv.n_pages;
        if (!in) atomicCAS(p.a.status, 0, 10 /* CATQ_ERR_INDEX */);
        row = in ? (id * kv.nkv + w.sh) * kv.page : kv.n_pages * kv.nkv * kv.page;  // (behind the last row: zeros)
      }
      if (!mbar_wait_warp(empty0 + 8u * slot, ph, p.wc)) return false;
      if (lane == 0) mbar_arrive_expect_tx(full0 + 8u * slot, static_cast<uint32_t>(pages * kv.page * HD));
      __syncwarp();
      if (lane < pages)
        tma_load_2d(base + Y::kOffRing + slot * Y::kTile + lane * kv.page * HD, map, full0 + 8u * slot, 0, row);
      ++loads;
      if (++slot == NS) { slot = 0; ph ^= 1u; }
      return true;
    };
    while (ok && w.next(g)) {
      // in the order in which the products take them
      ok = load(&tmk, 0) && (w.n < 2 || load(&tmk, 1));
      for (int32_t j = 0; ok && j < w.n; ++j) ok = load(&tmv, j) && (j + 2 >= w.n || load(&tmk, j + 2));
    }
    // copies still in flight land before the CTA exits
    for (int t = max(0, loads - NS); t < loads; ++t) drain(full0 + 8u * (t % NS), (t / NS) & 1);
  } else if (warp == kMmaWarp) {
    constexpr uint32_t kSwizzle = HD == 128 ? 2 : 4;
    constexpr uint32_t idesc_s = idesc_e4m3(kTok, NC, false, false), idesc_o = idesc_e4m3(HD, NC, true, true);
    constexpr uint32_t kHi = desc_hi(8 * HD, kSwizzle);  // code tiles: 8 rows of HD bytes from one group to the next
    constexpr uint32_t kHiQ = desc_hi(128, 0), kHiP = desc_hi(16 * kTok, 0);
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
        for (int k = 0; k < HD / 32; ++k)
          umma_f8(tmem + buf * NC, ad + 2 * k, kHi, bd + 2 * NC * k, kHiQ, idesc_s, k > 0 ? 1u : 0u);
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
          for (int k = 0; k < kTok / 32; ++k)
            umma_f8(tmem + kColO, ad + 2 * HD * k, kHi, bd + 32 * k, kHiP, idesc_o, (j > 0 || k > 0) ? 1u : 0u);
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
    // softmax: token tid of every tile
    const int tid = threadIdx.x;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    uint32_t gt = 0, ring = 0;  // tiles and loads before the segment's
    // page of the thread's token in tile t of the segment's sequence, -1 behind what is visible
    auto page_of = [&](int32_t t) -> int32_t {
      const int32_t tok = t * kTok + tid;
      if (t >= w.t0 + w.n || tok >= w.vis) return -1;
      const int32_t id = __ldg(kv.table + static_cast<int64_t>(w.sb) * kv.max_pages + tok / kv.page);
      return id < kv.n_pages ? id : -1;
    };
    auto scale_at = [&](const float* s, int32_t id) { return id < 0 ? 0.0f : __ldg(s + static_cast<int64_t>(id) * kv.nkv + w.sh); };
    // Products with the values up to tile t of the run have completed.  A barrier for every other tile: the scores of
    // tile t that the caller has seen followed the product of tile t - 2, so the barrier is at most one phase behind,
    // where a single one could be two behind and show the awaited parity.
    auto wait_pv = [&](uint32_t t) { return mbar_wait_warp(pv_done0 + 8u * (t & 1), (t >> 1) & 1, p.wc); };
    while (w.next(g)) {
      if (!bar_all(1, kSoft, ok)) { ok = false; break; }  // the rows' arrays are free
      const int32_t rows = min(R, w.ss.n * g.group - w.sq * R);
      int32_t id1 = page_of(w.t0);
      float ks1 = scale_at(kv.k_scale, id1), vs1 = scale_at(kv.v_scale, id1);
      id1 = page_of(w.t0 + 1);
      // queries: HD / 8 threads a row
      for (int r = tid / (HD / 8); r < R; r += kSoft / (HD / 8)) {
        const int i = tid % (HD / 8), row = w.sq * R + r;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows)
          v = *reinterpret_cast<const uint4*>(p.a.q + (w.ss.r0 + row / g.group) * p.a.ldq +
                                              (w.sh * g.group + row % g.group) * HD + 8 * i);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
        float x[8];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[2 * k] = __uint_as_float(u[k] << 16);
          x[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
          top = max(top, max(u[k] << 16 & 0x7fffffffu, u[k] & 0x7fff0000u));
        }
#pragma unroll
        for (int o = 1; o < HD / 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        // 2^-e brings the largest element into (224, 448]; a row that is not finite has NaN as its factor
        const int e = max(static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), -100);
        const bool bad = top >= 0x7f800000u;
        const float by = bad ? 0.0f : __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = bad ? 0.0f : x[k] * by;
        uint2 hi, lo;
        split8(x, hi, lo);
        // K-major without swizzle: 16 bytes of a row, the next 7 rows, the next rows' groups; then the next 16 bytes
        uint8_t* const at = gbase + Y::kOffQ + (i / 2) * (16 * NC) + (r / 8) * 128 + (r % 8) * 16 + (i % 2) * 8;
        *reinterpret_cast<uint2*>(at) = hi;
        *reinterpret_cast<uint2*>(at + 16 * R) = lo;
        if (i == 0) {
          row_f[r] = bad ? __uint_as_float(0x7fffffffu) : __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * p.a.scale_log2;
          row_m[r] = kNoMax;
          row_lim[r] = r < rows ? w.ss.len - w.ss.n + row / g.group : -1;
        }
      }
      fence_proxy_async_smem();
      soft_sync();
      if (lane == 0) mbar_arrive_local(q_full);
      const int32_t sees_all = row_lim[0] + 1;  // tokens that the first row sees, the others at least as many
      float l[R];
#pragma unroll
      for (int r = 0; r < R; ++r) l[r] = 0.0f;

      for (int32_t j = 0; j < w.n; ++j, ++gt) {
        const uint32_t buf = gt & 1;
        const float ks = ks1, vs = vs1;
        ks1 = scale_at(kv.k_scale, id1);
        vs1 = scale_at(kv.v_scale, id1);
        id1 = page_of(w.t0 + j + 2);
        const int32_t tok = (w.t0 + j) * kTok + tid;
        const bool masked = (w.t0 + j + 1) * kTok > sees_all;
        // log2 and reciprocal of the values' scale; codes under a scale of 0 are zeros, any scale serves them
        uint32_t vb = __float_as_uint(vs);
        if (vb == 0u) vb = (127u - 20u) << 23;
        const bool fin = vb < 0x7f800000u;
        const float lsv = fin ? static_cast<float>(static_cast<int>(vb >> 23) - 127) : vs;
        const float inv = fin ? __uint_as_float((254u - (vb >> 23)) << 23) : vs;
        ok = mbar_wait_warp(s_full0 + 8u * buf, (gt >> 1) & 1, p.wc) && ok;
        tc_fence_after();
        if (masked && (w.t0 + j + 1) * kTok > w.vis) {
          // the values behind the last visible token become zeros
          const uint32_t at = ring + min(2, w.n) + j + max(0, min(j, w.n - 2)), sl = at % NS;
          ok = mbar_wait_warp(full0 + 8u * sl, (at / NS) & 1, p.wc) && ok;
          const int32_t left = max(w.vis - (w.t0 + j) * kTok, 0);
          uint4* const v = reinterpret_cast<uint4*>(gbase + Y::kOffRing + sl * Y::kTile);
          for (int32_t i = left * (HD / 16) + tid; i < kTok * (HD / 16); i += kSoft) v[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        bool failed = false;
#pragma unroll
        for (int c = 0; c < R / CH; ++c) {
          uint32_t s[R < 16 ? 16 : 32];
          load_chunk<R>(lanes + buf * NC, c, s);
          float x[CH], m[CH];
          bool over = false;
#pragma unroll
          for (int i = 0; i < CH; ++i) {
            m[i] = row_m[c * CH + i];
            x[i] = fmaf(__uint_as_float(s[i + CH]), kLoUnit, __uint_as_float(s[i])) * (ks * row_f[c * CH + i]);
            const float y = x[i] + (lsv - m[i]);
            if (masked && tok > row_lim[c * CH + i]) x[i] = -INFINITY;
            else over |= y > kOver;
          }
          if (!bar_all(1, kSoft, ok && !over)) {
            if (!bar_all(1, kSoft, ok)) { failed = true; break; }
            // new maxima of the chunk's rows, and what they were worth before
#pragma unroll
            for (int i = 0; i < CH; ++i) {
              float t = x[i] + lsv;
#pragma unroll
              for (int o = 16; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
              if (lane == 0) red[warp * R + i] = t;
            }
            soft_sync();
            float f[CH];
            bool any = false;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
              const float t = fmaxf(fmaxf(red[i], red[R + i]), fmaxf(red[2 * R + i], red[3 * R + i]));
              const float raised = t - m[i] > kNominal ? t - kNominal : m[i];
              f[i] = raised == m[i] ? 1.0f : fast_exp2(m[i] - raised);
              any |= raised != m[i];
              m[i] = raised;
              l[c * CH + i] *= f[i];
            }
            if (j > 0 && any) {
              ok = wait_pv(gt - 1) && ok;
              tc_fence_after();
              uint32_t o[R < 16 ? 16 : 32];
              load_chunk<R>(lanes + kColO, c, o);
#pragma unroll
              for (int i = 0; i < CH; ++i) {
                o[i] = __float_as_uint(__uint_as_float(o[i]) * f[i]);
                o[i + CH] = __float_as_uint(__uint_as_float(o[i + CH]) * f[i]);
              }
              store_chunk<R>(lanes + kColO, c, o);
              tmem_st_wait();
            }
            soft_sync();  // everyone has read the old maxima and the parts of the new
            if (tid == 0) {
#pragma unroll
              for (int i = 0; i < CH; ++i) row_m[c * CH + i] = m[i];
            }
            soft_sync();
          }
          float wt[CH];
#pragma unroll
          for (int i = 0; i < CH; ++i) {
            wt[i] = fast_exp2(x[i] + (lsv - m[i]));
            if (masked) {
              const bool sees = tok <= row_lim[c * CH + i];
              wt[i] = sees ? wt[i] : 0.0f;
              l[c * CH + i] += sees ? wt[i] * inv : 0.0f;
            } else {
              l[c * CH + i] = fmaf(wt[i], inv, l[c * CH + i]);
            }
          }
          // MN-major without swizzle: 16 columns of a token, the next tokens; then the next 16 columns
          uint8_t* const at = gbase + Y::kOffP + buf * Y::kP + tid * 16;
          uint2 hi[CH / 8], lo[CH / 8];
#pragma unroll
          for (int i = 0; i < CH / 8; ++i) split8(wt + 8 * i, hi[i], lo[i]);
          if constexpr (R < 16) {
            *reinterpret_cast<uint4*>(at) = make_uint4(hi[0].x, hi[0].y, lo[0].x, lo[0].y);
          } else {
            *reinterpret_cast<uint4*>(at + c * (16 * kTok)) = make_uint4(hi[0].x, hi[0].y, hi[1].x, hi[1].y);
            *reinterpret_cast<uint4*>(at + (R / 16 + c) * (16 * kTok)) = make_uint4(lo[0].x, lo[0].y, lo[1].x, lo[1].y);
          }
        }
        if (failed) { ok = false; break; }
        tc_fence_before();
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_local(p_full0 + 8u * buf);
      }
      if (!bar_all(1, kSoft, ok)) { ok = false; break; }
      ring += 2 * w.n;

      // the rows' sums
      warp_row_sums<R>(l, lane);
      if constexpr (R >= 32) {
#pragma unroll
        for (int i = 0; i < R / 32; ++i) red[warp * R + lane * (R / 32) + i] = l[i];
      } else {
        if (lane % (32 / R) == 0) red[warp * R + lane / (32 / R)] = l[0];
      }
      soft_sync();
      ok = wait_pv(gt - 1);
      tc_fence_after();
      const bool whole = w.n == w.all;
      const int dl = HD == 128 ? tid : warp * 16 + lane;  // the thread's column of the head (64: lanes 0 .. 15)
      const bool mine = HD == 128 || lane < 16;
      float* const part = p.parts + (2 * static_cast<int64_t>(blockIdx.x) + (w.begin >= first ? 1 : 0)) * Y::kPartFloats;
#pragma unroll
      for (int c = 0; c < R / CH; ++c) {
        uint32_t o[R < 16 ? 16 : 32];
        load_chunk<R>(lanes + kColO, c, o);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const int r = c * CH + i;
          if (!ok || !mine || r >= rows) continue;
          const float v = fmaf(__uint_as_float(o[i + CH]), kLoUnit, __uint_as_float(o[i]));
          if (whole) {
            const float sum = (red[r] + red[R + r]) + (red[2 * R + r] + red[3 * R + r]);
            const int row = w.sq * R + r;
            const __nv_bfloat16 out = __float2bfloat16_rn(sum == 0.0f ? 0.0f : v / sum);
            p.a.o[(w.ss.r0 + row / g.group) * p.a.ldo + (w.sh * g.group + row % g.group) * HD + dl] =
                *reinterpret_cast<const uint16_t*>(&out);
          } else {
            part[2 * R + r * HD + dl] = v;
          }
        }
      }
      tc_fence_before();
      if (ok && tid < rows) {
        const float sum = (red[tid] + red[R + tid]) + (red[2 * R + tid] + red[3 * R + tid]);
        const int row = w.sq * R + tid;
        if (!whole) {
          part[tid] = row_m[tid];
          part[R + tid] = sum;
        } else if (p.a.lse) {
          p.a.lse[static_cast<int64_t>(w.ss.r0 + row / g.group) * p.a.nh + w.sh * g.group + row % g.group] =
              sum == 0.0f ? -INFINITY : (row_m[tid] + log2f(sum)) * 0.6931471805599453f;
        }
      }
      if (whole) continue;
      // the last of the row tile's runs joins their parts
      if (!bar_all(1, kSoft, ok)) { ok = false; break; }
      const int32_t c0 = static_cast<int32_t>(w.begin / run), c1 = static_cast<int32_t>((w.begin + w.all - 1) / run);
      __threadfence();
      soft_sync();
      if (tid == 0) {
        const uint32_t last = static_cast<uint32_t>(c1 - c0);
        *merge_flag = atomicInc(p.counters + c0, last) == last;
      }
      soft_sync();
      if (*merge_flag) {
        __threadfence();
        constexpr int kLanes = HD / 4;  // threads a row
        for (int r = tid / kLanes; r < rows; r += kSoft / kLanes) {
          const int i = tid % kLanes;
          float m = kNoMax, sum = 0.0f, o[4] = {0.f, 0.f, 0.f, 0.f};
          for (int32_t c = c0; c <= c1; c += 8) {
            float pm[8], pl[8];
            float4 po[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float* const q = p.parts + (2 * static_cast<int64_t>(min(c + k, c1)) + (c + k == c0 ? 1 : 0)) * Y::kPartFloats;
              pm[k] = __ldcg(q + r);
              pl[k] = c + k <= c1 ? __ldcg(q + R + r) : 0.0f;
              po[k] = __ldcg(reinterpret_cast<const float4*>(q + 2 * R + r * HD) + i);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (c + k <= c1) {
                const float top = fmaxf(m, pm[k]), f = fast_exp2(m - top), e = fast_exp2(pm[k] - top);
                sum = sum * f + pl[k] * e;
                o[0] = o[0] * f + po[k].x * e;
                o[1] = o[1] * f + po[k].y * e;
                o[2] = o[2] * f + po[k].z * e;
                o[3] = o[3] * f + po[k].w * e;
                m = top;
              }
          }
          const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
          const int row = w.sq * R + r;
          const int64_t tk = w.ss.r0 + row / g.group, hd = w.sh * g.group + row % g.group;
          uint2 out;
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(out.x) : "f"(o[1] * by), "f"(o[0] * by));
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(out.y) : "f"(o[3] * by), "f"(o[2] * by));
          *reinterpret_cast<uint2*>(p.a.o + tk * p.a.ldo + hd * HD + 4 * i) = out;
          if (p.a.lse && i == 0)
            p.a.lse[tk * p.a.nh + hd] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc<1>(tmem, Y::kTmem);
  }
}

PFN_cuTensorMapEncodeTiled_v12000 g_enc = nullptr;
std::once_flag g_enc_once;

// Codes as [n_pages n_kv_heads page] rows of d bytes, boxes of one page and head, rows swizzled over their own length.
bool tmap_codes(CUtensorMap* m, const void* ptr, int32_t d, int64_t rows, int32_t page) {
  std::call_once(g_enc_once, [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q{};
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      g_enc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  });
  if (!g_enc) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(d)};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(d), static_cast<cuuint32_t>(page)};
  const cuuint32_t estr[2] = {1, 1};
  return g_enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count() {
  int sm = 152, dev = 0;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev);
  return sm;
}

constexpr size_t kCounterBytes = 4096;  // up to 1024 CTAs

template <int HD, int R>
cudaError_t run_kv(const KvAttnArgs& a, cudaStream_t st) {
  using Y = KvLay<HD, R>;
  CUtensorMap tk, tv;
  const int64_t rows = static_cast<int64_t>(a.cache.n_pages) * a.cache.nkv * a.cache.page;
  if (!tmap_codes(&tk, a.cache.k_codes, HD, rows, a.cache.page) || !tmap_codes(&tv, a.cache.v_codes, HD, rows, a.cache.page))
    return cudaErrorInvalidValue;
  KvTcArgs p{};
  p.a = a;
  if (!launch_wait_ctl(&p.wc)) return cudaErrorInvalidDevice;
  p.a.status = p.wc.status_word;
  p.g = KvGeom{a.row_start, a.seq_len, a.B, a.nh / a.cache.nkv, a.cache.nkv, a.T,
               static_cast<int64_t>(a.cache.max_pages) * a.cache.page};
  p.counters = static_cast<uint32_t*>(a.workspace);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + kCounterBytes);
  p.min_run = 2;
  auto kern = kv_attn_kernel<HD, R>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Y::kSmem);
  if (e != cudaSuccess) return e;
  kern<<<static_cast<unsigned>(std::min(Y::kCtas * sm_count(), 1024)), kThreads, Y::kSmem, st>>>(tk, tv, p);
  return cudaGetLastError();
}

// Rows of a tile: what an average sequence has a key/value head (any number is right).
template <int HD>
cudaError_t run_kv_rows(const KvAttnArgs& a, cudaStream_t st) {
  const int64_t rows = (a.T + a.B - 1) / a.B * (a.nh / a.cache.nkv);
  if (rows <= 8) return run_kv<HD, 8>(a, st);
  if (rows <= 16) return run_kv<HD, 16>(a, st);
  if (rows <= 32) return run_kv<HD, 32>(a, st);
  return run_kv<HD, 64>(a, st);
}

}  // namespace

size_t kv_attention_ws_bytes(int32_t, int32_t, int32_t d) {
  // two parts of up to 32 rows for each of two CTAs an SM, or of 64 for one
  const size_t ctas = static_cast<size_t>(std::min(2 * sm_count(), 1024));
  const size_t parts = ctas * 2 * 32 * (static_cast<size_t>(d) + 2) * sizeof(float);
  return (kCounterBytes + parts + 255) / 256 * 256;
}

cudaError_t launch_kv_attention(KvAttnArgs a, cudaStream_t st) {
  return a.cache.d == 128 ? run_kv_rows<128>(a, st) : run_kv_rows<64>(a, st);
}

}  // namespace catq
