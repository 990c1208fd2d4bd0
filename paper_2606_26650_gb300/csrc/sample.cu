// sample.cu — a token for each row of logits from a given random number (catq_sample): temperature, top-k, top-p and
// min-p.
//
// A token weighs w = rint(2^40 exp((x - max) / T)), a whole number: sums do not depend on the order of their terms, and
// every comparison (does the cumulated weight reach p of the whole, does it pass u of what is kept) is one of integers.
// The order is by falling x, ties by rising index, so that each filter leaves a first part of it and the drawn token is
// the first whose cumulated weight passes floor(u Z).  Nothing is sorted: a first part's end is found by a histogram of
// counts and weights over the range of keys (x's bits as a number that rises as x falls) that have any weight, then
// inside one of its bins: by ranks where it has few tokens, by a finer histogram where it has many.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "launch.h"

namespace catq {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kBinBits = 12, kBins = 1 << kBinBits;
constexpr int kList = 1024;  // tokens whose ranks are found one against all others

// ---------------------------------------------------------------- weights
// 2^(-i / 64) in units of 2^-63.
__device__ const uint64_t kPow2[64] = {
    0x8000000000000000ull, 0x7e9f06067a4360baull, 0x7d41d96db915019dull, 0x7be86fb985689ddcull,
    0x7a92be8a92436616ull, 0x7940bb9e2cffd89dull, 0x77f25ccdee6d7ae6ull, 0x76a7980f6cca15c2ull,
    0x75606373ee921c97ull, 0x741cb5281e25ee34ull, 0x72dc8373be41a454ull, 0x719fc4b95f452d29ull,
    0x70666f76154a7089ull, 0x6f307a412f074892ull, 0x6dfddbcbed791babull, 0x6cce8ae13c57ebdbull,
    0x6ba27e656b4eb57aull, 0x6a79ad55e7f6fd10ull, 0x69540ec8f895722dull, 0x683199ed779592caull,
    0x6712460a8fc24072ull, 0x65f60a7f79393e2eull, 0x64dcdec3371793d1ull, 0x63c6ba6455dcd8aeull,
    0x62b39508aa836d6full, 0x61a3666d124bb204ull, 0x6096266533384a2bull, 0x5f8bccdb3d398841ull,
    0x5e8451cfac061b5full, 0x5d7fad59099f22feull, 0x5c7dd7a3b17dcf75ull, 0x5b7ec8f19468bbc9ull,
    0x5a827999fcef3242ull, 0x5988e20954889245ull, 0x5891fac0e95612c8ull, 0x579dbc56b48521baull,
    0x56ac1f752150a563ull, 0x55bd1cdad49f699cull, 0x54d0ad5a753e077cull, 0x53e6c9da74b29ab5ull,
    0x52ff6b54d8a89c75ull, 0x521a8ad704f3404full, 0x513821818624b40cull, 0x50582887dcb8a7e1ull,
    0x4f7a993048d088d7ull, 0x4e9f6cd3967fdba8ull, 0x4dc69cdceaa72a9cull, 0x4cf022c9905bfd32ull,
    0x4c1bf828c6dc54b8ull, 0x4b4a169b900c2d00ull, 0x4a7a77d47f7b84b1ull, 0x49ad159789f37496ull,
    0x48e1e9b9d588e19bull, 0x4818ee218a3358eeull, 0x47521cc5a2e6a9e0ull, 0x468d6fadbf2dd4f3ull,
    0x45cae0f1f545eb73ull, 0x450a6abaa4b77ecdull, 0x444c0740496d4294ull, 0x438fb0cb4f468808ull,
    0x42d561b3e6243d8aull, 0x421d1461d66f2023ull, 0x4166c34c5615d0ecull, 0x40b268f9de0183baull};
constexpr int kOneBits = 40;                     // the largest weight is 2^40
constexpr uint64_t kOne = uint64_t(1) << kOneBits;

// Weights of a row: exp(-(max - x) / T) as 2^-t in integers, t = D C / 2^64 in units of 2^-56 with D = (max - x) 2^k, which has
// up to 63 bits (max - x as an fp32 number and its rounding, both exact), and C = 2^(120 - k) log2(e) / T.  t is its whole part,
// its next six bits (a table) and a rest below 2^-6, whose exponential is its series up to y^5 / 5!, y < 2^-6.5 (remainder
// 2^-48.6).  What is cut off in C (53 bits) and the products leaves a weight within 2^-44 of itself before it is rounded.
struct Weigher {
  float max, cut, scale;  // max - x at and above cut weighs nothing
  uint64_t c;
  const uint64_t* pow2;
  __device__ __forceinline__ uint64_t operator()(float x) const {
    const float d = max - x;
    if (!(d < cut)) return 0;
    const float b = d - max, rest = (max - (d - b)) + (-x - b);
    const uint64_t big = static_cast<uint64_t>(__float2ll_rn(d * scale) + __float2ll_rn(rest * scale));
    const uint64_t t = __umul64hi(big, c);
    const int n = static_cast<int>(t >> 56);
    if (n > kOneBits) return 0;
    const uint64_t p = pow2[(t >> 50) & 63];
    const uint64_t y = __umul64hi(t << 14, 0xb17217f7d1cf79acull);  // ln 2 of the rest: 64 y
    const uint32_t h = static_cast<uint32_t>(y >> 32);
    // (1 - e^-y) / y = 1 - y/2 (1 - y/3 (1 - y/4 (1 - y/5)))
    uint32_t q = 0xffffffffu - __umulhi(h, 0x00cccccdu);
    q = 0xffffffffu - (__umulhi(h, q) >> 8);
    q = 0xffffffffu - __umulhi(__umulhi(h, q), 0x01555555u);
    const uint64_t s = ~(__umul64hi(y, static_cast<uint64_t>(q) << 32) >> 7);
    const uint64_t e = p - __umul64hi(p, __umul64hi(y, s) >> 6);
    const int down = 63 - kOneBits + n;
    return (e + (uint64_t(1) << (down - 1))) >> down;
  }
};

// The weights of a row with largest logit `max` at temperature t > 0.
__device__ __forceinline__ Weigher weigher(float max, float t, const uint64_t* pow2) {
  const double rate = 1.4426950408889634 / fmin(fmax(static_cast<double>(t), 0x1p-60), 0x1p60);
  int e;
  frexp(41.5 / rate, &e);
  Weigher w;
  w.max = max;
  w.cut = static_cast<float>(41.2 / rate);
  w.scale = static_cast<float>(ldexp(1.0, 63 - e));
  w.c = static_cast<uint64_t>(ldexp(rate, 57 + e));
  w.pow2 = pow2;
  return w;
}

// ---------------------------------------------------------------- logits
// Keys rise as x falls; both zeros have one.
template <typename E>
struct Logit;
template <>
struct Logit<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ uint32_t key(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? u : ~u & 0x7fffffffu;
  }
  static __device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k : ~k & 0x7fffffffu); }
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  static __device__ __forceinline__ void get(const uint4& q, float* x) {
    x[0] = __uint_as_float(q.x);
    x[1] = __uint_as_float(q.y);
    x[2] = __uint_as_float(q.z);
    x[3] = __uint_as_float(q.w);
  }
};
template <>
struct Logit<uint16_t> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ uint32_t key(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f) >> 16;
    return u & 0x8000u ? u : ~u & 0x7fffu;
  }
  static __device__ __forceinline__ float of_key(uint32_t k) {
    return __uint_as_float((k & 0x8000u ? k : ~k & 0x7fffu) << 16);
  }
  static __device__ __forceinline__ float get(const uint16_t* p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }
  static __device__ __forceinline__ void get(const uint4& q, float* x) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};

// A row: elements up to the first 16-byte boundary, vectors, elements behind the last one.
template <typename E>
struct Row {
  const E* p;
  int32_t V, head, vecs;
  __device__ __forceinline__ Row(const E* row, int32_t n) : p(row), V(n) {
    head = min(V, static_cast<int32_t>((16u - (reinterpret_cast<uintptr_t>(row) & 15u)) % 16u / sizeof(E)));
    vecs = (V - head) / Logit<E>::kVec;
  }
  __device__ __forceinline__ const uint4* vec() const { return reinterpret_cast<const uint4*>(p + head); }
  __device__ __forceinline__ int32_t tail() const { return head + vecs * Logit<E>::kVec; }
  // f(x, index) of every element, by the CTA's threads.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    constexpr int VEC = Logit<E>::kVec;
    const int32_t t = threadIdx.x;
    if (t < head) f(Logit<E>::get(p + t), t);
    for (int32_t v = t; v < vecs; v += kThreads) {
      float x[VEC];
      Logit<E>::get(vec()[v], x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f(x[i], head + v * VEC + i);
    }
    if (tail() + t < V) f(Logit<E>::get(p + tail() + t), tail() + t);
  }
};

// ---------------------------------------------------------------- histograms
// Counts and weights by bins; after sum_up those of a bin and all before it.
struct Bins {
  uint32_t count[kBins], lo[kBins], hi[kBins];
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < kBins; i += kThreads) count[i] = lo[i] = hi[i] = 0;
  }
  __device__ __forceinline__ void add(int bin, uint64_t w) {
    atomicAdd(&count[bin], 1u);
    const uint32_t low = static_cast<uint32_t>(w), old = atomicAdd(&lo[bin], low);
    const uint32_t high = static_cast<uint32_t>(w >> 32) + (old + low < old ? 1u : 0u);
    if (high) atomicAdd(&hi[bin], high);
  }
  __device__ __forceinline__ uint64_t weight(int bin) const { return static_cast<uint64_t>(hi[bin]) << 32 | lo[bin]; }
};

struct Shared {
  Bins bins[2];
  uint64_t pow2[64];
  uint64_t list_w[kList];
  uint32_t list_key[kList];
  int32_t list_at[kList];
  uint64_t red_w[kWarps];
  uint32_t red_c[kWarps];
  uint32_t n;
  // a place in the order
  uint32_t key, before;      // its key and how many are ahead of it
  uint64_t w, w_before;      // its weight and theirs
  int32_t at;                // its index, where it was asked for
  Weigher weigh;
};

// Sums over the CTA (in every thread), counts and weights.
__device__ __forceinline__ void block_sums(Shared& s, uint32_t& c, uint64_t& w) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    c += __shfl_xor_sync(0xffffffffu, c, o);
    w += __shfl_xor_sync(0xffffffffu, w, o);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) {
    s.red_c[threadIdx.x >> 5] = c;
    s.red_w[threadIdx.x >> 5] = w;
  }
  __syncthreads();
  c = 0;
  w = 0;
  for (int i = 0; i < kWarps; ++i) {
    c += s.red_c[i];
    w += s.red_w[i];
  }
}

// Bins to running sums, on top of what came before them.
__device__ __forceinline__ void sum_up(Shared& s, Bins& b, uint32_t c0, uint64_t w0) {
  constexpr int kPer = kBins / kThreads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t c[kPer];
  uint64_t w[kPer];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = threadIdx.x * kPer + i;
    c[i] = b.count[at] + (i ? c[i - 1] : 0u);
    w[i] = b.weight(at) + (i ? w[i - 1] : 0u);
  }
  uint32_t cs = c[kPer - 1];
  uint64_t ws = w[kPer - 1];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, cs, o);
    const uint64_t y = __shfl_up_sync(0xffffffffu, ws, o);
    if (lane >= o) {
      cs += x;
      ws += y;
    }
  }
  if (lane == 31) {
    s.red_c[warp] = cs;
    s.red_w[warp] = ws;
  }
  __syncthreads();
  uint32_t cb = c0 + cs - c[kPer - 1];
  uint64_t wb = w0 + ws - w[kPer - 1];
  for (int i = 0; i < warp; ++i) {
    cb += s.red_c[i];
    wb += s.red_w[i];
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = threadIdx.x * kPer + i;
    const uint64_t v = wb + w[i];
    b.count[at] = cb + c[i];
    b.lo[at] = static_cast<uint32_t>(v);
    b.hi[at] = static_cast<uint32_t>(v >> 32);
  }
  __syncthreads();
}

// The first bin whose running sum reaches target >= 1.
__device__ __forceinline__ int first_bin(const Bins& b, bool by_weight, uint64_t target) {
  int lo = 0, hi = kBins - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if ((by_weight ? b.weight(mid) : b.count[mid]) >= target)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// ---------------------------------------------------------------- a place in the order
// The j-th element of a row (from 0) that has the key, in the order of the indexes, into s.at.
template <typename E>
__device__ __forceinline__ void nth_of(Shared& s, const Row<E>& row, uint32_t key, uint32_t j) {
  constexpr int VEC = Logit<E>::kVec;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t seen = 0;
  // x: n consecutive elements of the thread from index `at` on, the threads' in order
  auto step = [&](const float* x, int n, int32_t at) {
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) mine += i < n && Logit<E>::key(x[i]) == key ? 1u : 0u;
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    __syncthreads();
    if (lane == 31) s.red_c[warp] = upto;
    __syncthreads();
    uint32_t base = seen;
    for (int i = 0; i < kWarps; ++i) {
      if (i == warp) upto += base;
      base += s.red_c[i];
    }
    uint32_t before = upto - mine;
    if (before <= j && j < upto) {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (i < n && Logit<E>::key(x[i]) == key) {
          if (before == j) s.at = at + i;
          ++before;
        }
    }
    seen = base;
  };
  float x[VEC];
  x[0] = static_cast<int>(threadIdx.x) < row.head ? Logit<E>::get(row.p + threadIdx.x) : 0.0f;
  step(x, static_cast<int>(threadIdx.x) < row.head ? 1 : 0, threadIdx.x);
  for (int32_t v0 = 0; v0 < row.vecs && seen <= j; v0 += kThreads) {
    const int32_t v = v0 + threadIdx.x;
    if (v < row.vecs) Logit<E>::get(row.vec()[v], x);
    step(x, v < row.vecs ? VEC : 0, row.head + v * VEC);
  }
  if (seen <= j) {
    const int32_t at = row.tail() + threadIdx.x;
    if (at < row.V) x[0] = Logit<E>::get(row.p + at);
    step(x, at < row.V ? 1 : 0, at);
  }
  __syncthreads();
}

// The first place at which the running count or weight reaches target >= 1, which the row has.  first: the key of the
// largest logit, shift: bins[0] holds the running sums over bins of 2^shift keys from there on.
template <typename E>
__device__ __forceinline__ void find(Shared& s, const Row<E>& row, uint32_t first, int shift, bool by_weight, uint64_t target,
                                     bool want_at) {
  uint32_t lo = 0, c0 = 0, n;
  uint64_t w0 = 0;
  const Bins* b = &s.bins[0];
  for (;;) {
    const int bin = first_bin(*b, by_weight, target);
    if (bin > 0) {
      c0 = b->count[bin - 1];
      w0 = b->weight(bin - 1);
    }
    n = b->count[bin] - c0;
    lo += static_cast<uint32_t>(bin) << shift;
    __syncthreads();
    if (shift == 0) {
      const uint64_t w = s.weigh(Logit<E>::of_key(first + lo));
      const uint32_t j = static_cast<uint32_t>(by_weight ? (target - w0 - 1) / w : target - c0 - 1);
      if (threadIdx.x == 0) {
        s.key = first + lo;
        s.before = c0 + j;
        s.w = w;
        s.w_before = w0 + j * w;
      }
      if (want_at) nth_of(s, row, first + lo, j);
      __syncthreads();
      return;
    }
    if (n <= kList) break;
    const int finer = max(shift - kBinBits, 0);
    s.bins[1].clear();
    __syncthreads();
    row.each([&](float x, int32_t) {
      const uint32_t rel = Logit<E>::key(x) - first - lo;
      if (rel >> shift) return;
      const uint64_t w = s.weigh(x);
      if (w) s.bins[1].add(rel >> finer, w);
    });
    sum_up(s, s.bins[1], c0, w0);
    shift = finer;
    b = &s.bins[1];
  }
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  row.each([&](float x, int32_t at) {
    const uint32_t k = Logit<E>::key(x);
    if ((k - first - lo) >> shift) return;
    const uint64_t w = s.weigh(x);
    if (!w) return;
    const uint32_t i = atomicAdd(&s.n, 1u);
    if (i >= kList) return;
    s.list_key[i] = k;
    s.list_at[i] = at;
    s.list_w[i] = w;
  });
  __syncthreads();
  const uint32_t m = min(s.n, static_cast<uint32_t>(kList));
  for (uint32_t e = threadIdx.x; e < m; e += kThreads) {
    const uint32_t k = s.list_key[e];
    const int32_t at = s.list_at[e];
    uint32_t c = c0;
    uint64_t w = w0;
    for (uint32_t i = 0; i < m; ++i) {
      const uint32_t ki = s.list_key[i];
      if (ki < k || (ki == k && s.list_at[i] < at)) {
        ++c;
        w += s.list_w[i];
      }
    }
    const uint64_t mine = by_weight ? w : c, with = mine + (by_weight ? s.list_w[e] : 1u);
    if (mine < target && target <= with) {
      s.key = k;
      s.before = c;
      s.w = s.list_w[e];
      s.w_before = w;
      s.at = at;
    }
  }
  __syncthreads();
}

// One CTA a row.
template <typename E>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a) {
  extern __shared__ uint8_t smem_raw[];
  Shared& s = *reinterpret_cast<Shared*>(smem_raw);
  const int64_t r = blockIdx.x;
  const Row<E> row(static_cast<const E*>(a.logits) + r * a.ld, a.V);
  if (threadIdx.x < 64) s.pow2[threadIdx.x] = kPow2[threadIdx.x];
  s.bins[0].clear();

  // the largest logit, as the least key; not a number, or +inf, is worse than any
  uint32_t best = 0xffffffffu, bad = 0;
  row.each([&](float x, int32_t) {
    bad |= x < INFINITY ? 0u : 1u;
    best = min(best, Logit<E>::key(x));
  });
  best = __reduce_min_sync(0xffffffffu, best);
  bad = __syncthreads_or(bad);
  if ((threadIdx.x & 31) == 0) s.red_c[threadIdx.x >> 5] = best;
  __syncthreads();
  for (int i = 0; i < kWarps; ++i) best = min(best, s.red_c[i]);
  const float max = Logit<E>::of_key(best);
  const float t = a.temperature ? a.temperature[r] : 1.0f;
  if (bad || max == -INFINITY || !(t >= 0.0f)) {  // nothing can be drawn
    if (threadIdx.x == 0) {
      a.tokens[r] = -1;
      if (a.logprob) a.logprob[r] = __uint_as_float(0x7fffffffu);
    }
    return;
  }
  const bool greedy = t == 0.0f;
  if (threadIdx.x == 0) s.weigh = weigher(max, greedy ? 1.0f : t, s.pow2);
  __syncthreads();

  // all tokens that weigh anything
  const uint32_t range = Logit<E>::key(fmaxf(__fsub_rd(max, 1.001f * s.weigh.cut), -3.402823466e38f)) - best;
  int shift = 0;
  while (range >> shift >= kBins) ++shift;
  row.each([&](float x, int32_t) {
    const uint64_t w = s.weigh(x);
    if (w) s.bins[0].add(min((Logit<E>::key(x) - best) >> shift, kBins - 1u), w);
  });
  sum_up(s, s.bins[0], 0, 0);
  const uint32_t live = s.bins[0].count[kBins - 1];

  // what is kept: the first `kept` tokens, weighing `total` together
  uint32_t kept = live;
  uint64_t total = s.bins[0].weight(kBins - 1);
  auto limit = [&] {  // up to the place found, with it
    if (s.before + 1 < kept) {
      kept = s.before + 1;
      total = s.w_before + s.w;
    }
    __syncthreads();
  };
  const int32_t k = greedy ? 1 : a.top_k ? a.top_k[r] : 0;
  if (k > 0 && static_cast<uint32_t>(k) < live) {
    find(s, row, best, shift, false, k, false);
    limit();
  }
  const float p = a.top_p && !greedy ? a.top_p[r] : 1.0f;
  const float least = a.min_p && !greedy ? a.min_p[r] : 0.0f;
  if (p < 1.0f) {
    const double part = ceil(static_cast<double>(p) * static_cast<double>(total));
    const uint64_t need = part < 1.0 ? 1u : part < static_cast<double>(total) ? static_cast<uint64_t>(part) : total;
    find(s, row, best, shift, true, need, false);
    limit();
  }
  if (least > 0.0f) {
    const uint64_t w0 = static_cast<uint64_t>(ceil(static_cast<double>(fminf(least, 1.0f)) * static_cast<double>(kOne)));
    uint32_t c = 0;
    uint64_t sum = 0;
    row.each([&](float x, int32_t) {
      const uint64_t w = s.weigh(x);
      if (w >= w0) {
        ++c;
        sum += w;
      }
    });
    block_sums(s, c, sum);
    if (c < kept) {
      kept = c;
      total = sum;
    }
    __syncthreads();
  }

  // the first whose running weight passes u of the whole
  const double part = floor(static_cast<double>(a.u[r]) * static_cast<double>(total));
  const uint64_t pass = !(part > 0.0) ? 0u : part < static_cast<double>(total - 1) ? static_cast<uint64_t>(part) : total - 1;
  find(s, row, best, shift, true, pass + 1, true);
  if (threadIdx.x == 0) {
    a.tokens[r] = s.at;
    if (a.logprob) {  // ln(w / total), where w is most of it from what is left
      const float rest = static_cast<float>(total - s.w) / static_cast<float>(total);
      a.logprob[r] = rest < 0.5f ? log1pf(-rest) : logf(static_cast<float>(s.w) / static_cast<float>(total));
    }
  }
}

template <typename E>
cudaError_t run_sample(const SampleArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};  // devices on which the kernel may use its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(sample_kernel<E>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(Shared)));
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  sample_kernel<E><<<static_cast<unsigned>(a.R), kThreads, sizeof(Shared), st>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, bool f32, cudaStream_t st) {
  return f32 ? run_sample<float>(a, st) : run_sample<uint16_t>(a, st);
}

}  // namespace catq
