// sample.cu — a token for each row of logits from a given random number (catq_sample): temperature, top-k, top-p and
// min-p.
//
// A token weighs w = rint(2^40 exp((x - max) / T)), a whole number: sums do not depend on the order of their terms, and
// every comparison (does the cumulated weight reach p of the whole, does it pass u of what is kept) is one of integers.
// The order is by falling x, ties by rising index, so that each filter leaves a first part of it and the drawn token is
// the first whose cumulated weight passes floor(u Z).  Nothing is sorted: a first part's end is found by a histogram of
// counts and weights over the range of keys (x's bits as a number that rises as x falls) that have any weight, then
// inside one of its bins: by ranks where it has few tokens, by a finer histogram where it has many.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "launch.h"
#include "ptx_sm100.cuh"

namespace catq {
namespace {

namespace cg = cooperative_groups;

constexpr float kLowest = -3.402823466e38f;
constexpr int32_t kTaken = -2;      // a row's token where a cluster of the second kernel has taken it,
constexpr int32_t kUndecided = -3;  // where the first kernel leaves it to the second, and below that where
// the first kernel leaves it and knows that its tokens can be drawn and which is the largest.
__device__ __forceinline__ int32_t left_with(int32_t at) { return at <= 0x7ffffffc ? kUndecided - 1 - at : kUndecided; }
__device__ __forceinline__ int32_t largest_of(int32_t left) { return kUndecided - 1 - left; }  // -1: not known

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

// Weights of a row: exp(-(max - x) / T) as 2^-t in integers, t = D C / 2^64 in units of 2^-56 with D = (max - x) 2^k, which has
// up to 63 bits (max - x as an fp32 number and its rounding, both exact), and C = 2^(120 - k) log2(e) / T.  t is its whole part,
// its next six bits (a table) and a rest below 2^-6, whose exponential is its series up to y^5 / 5!, y < 2^-6.5 (remainder
// 2^-48.6).  What is cut off in C (53 bits) and the products leaves a weight within 2^-44 of itself before it is rounded.
// 2^-f of the fraction f of t (units of 2^-56), in units of 2^-63.
__device__ __forceinline__ uint64_t exp2_fraction(uint64_t t, const uint64_t* pow2) {
  const uint64_t p = pow2[(t >> 50) & 63];
  const uint64_t y = __umul64hi(t << 14, 0xb17217f7d1cf79acull);  // ln 2 of the rest: 64 y
  const uint32_t h = static_cast<uint32_t>(y >> 32);
  // (1 - e^-y) / y = 1 - y/2 (1 - y/3 (1 - y/4 (1 - y/5)))
  uint32_t q = 0xffffffffu - __umulhi(h, 0x00cccccdu);
  q = 0xffffffffu - (__umulhi(h, q) >> 8);
  q = 0xffffffffu - __umulhi(__umulhi(h, q), 0x01555555u);
  const uint64_t s = ~(__umul64hi(y, static_cast<uint64_t>(q) << 32) >> 7);
  return p - __umul64hi(p, __umul64hi(y, s) >> 6);
}

__device__ __forceinline__ uint64_t weight_inline(float d, float rest, float scale, uint64_t c, const uint64_t* pow2) {
  const uint64_t big = static_cast<uint64_t>(__float2ll_rn(d * scale) + __float2ll_rn(rest * scale));
  const uint64_t t = __umul64hi(big, c);
  const int n = static_cast<int>(t >> 56);
  const int down = 63 - kOneBits + min(n, kOneBits);
  return n > kOneBits ? 0 : (exp2_fraction(t, pow2) + (uint64_t(1) << (down - 1))) >> down;
}
// (A call where a thread has few of them: code that is fetched for the first time costs a short kernel more than the call.)
__device__ __noinline__ uint64_t weight_of(float d, float rest, float scale, uint64_t c, const uint64_t* pow2) {
  return weight_inline(d, rest, scale, c, pow2);
}
struct Weigher {
  float max, cut, scale;  // max - x at and above cut weighs nothing
  uint64_t c;
  const uint64_t* pow2;
  __device__ __forceinline__ uint64_t operator()(float x) const {
    const float d = max - x;
    if (!(d < cut)) return 0;
    const float b = d - max;
    return weight_of(d, (max - (d - b)) + (-x - b), scale, c, pow2);
  }
  // The same beside others of its kind.
  __device__ __forceinline__ uint64_t beside(float x) const {
    const float d = max - x, held = fminf(d, cut), b = d - max;
    const uint64_t w = weight_inline(held, d < cut ? (max - (d - b)) + (-x - b) : 0.0f, scale, c, pow2);
    return d < cut ? w : 0;
  }
};

// The weights of a row with largest logit `max` at temperature t > 0.
__device__ __forceinline__ Weigher weigher(float max, float t, const uint64_t* pow2) {
  const float held = fminf(fmaxf(t, 0x1p-60f), 0x1p60f);
  const double wide = static_cast<double>(held), rate = 1.4426950408889634 / wide;
  // e: 41.5 / rate = 28.7655 t is below 2^e, by a factor of two at most
  const uint32_t most = __float_as_uint(28.7655830f * held);
  const int e = static_cast<int>(most >> 23) - 126 + ((most & 0x7fffffu) >= 0x7ffff0u ? 1 : 0);
  Weigher w;
  w.max = max;
  w.cut = 28.5576391f * held;  // 41.2 / rate
  w.scale = __uint_as_float(static_cast<uint32_t>(127 + 63 - e) << 23);
  w.c = static_cast<uint64_t>(__longlong_as_double(__double_as_longlong(rate) + (static_cast<int64_t>(57 + e) << 52)));
  w.pow2 = pow2;
  return w;
}

// The running weight at which p of the whole is reached: ceil(p whole), from 1 to whole.
__device__ __forceinline__ uint64_t reaches(float p, uint64_t whole) {
  const double part = ceil(static_cast<double>(p) * static_cast<double>(whole));
  return part < 1.0 ? 1 : part < static_cast<double>(whole) ? static_cast<uint64_t>(part) : whole;
}
// The least weight that min-p keeps.
__device__ __forceinline__ uint64_t least_of(float min_p) {
  return __float2ull_ru(fminf(min_p, 1.0f) * 0x1p40f);  // (an exact product)
}
// The running weight that the token has to reach: floor(u whole) + 1, from 1 to whole.
__device__ __forceinline__ uint64_t passes(float u, uint64_t whole) {
  const double part = floor(static_cast<double>(u) * static_cast<double>(whole));
  return (!(part > 0.0) ? 0 : part < static_cast<double>(whole - 1) ? static_cast<uint64_t>(part) : whole - 1) + 1;
}
// ln(w / whole); where w is most of it, by what is left.
__device__ __forceinline__ float ln_of(uint64_t w, uint64_t whole) {
  const float rest = static_cast<float>(whole - w) / static_cast<float>(whole);
  return rest < 0.5f ? log1pf(-rest) : logf(static_cast<float>(w) / static_cast<float>(whole));
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
  static __device__ __forceinline__ float get(const uint4& q, int e) {
    return __uint_as_float(e & 2 ? (e & 1 ? q.w : q.z) : (e & 1 ? q.y : q.x));
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
  static __device__ __forceinline__ float get(const uint4& q, int e) {
    const uint32_t w = e & 4 ? (e & 2 ? q.w : q.z) : (e & 2 ? q.y : q.x);
    return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
  }
};

// A row: elements up to the first 16-byte boundary, vectors, elements behind the last one.  In parts: part i of n has the
// vectors v0 .. v1 - 1, the first part the elements ahead of them, the last those behind.
template <typename E>
struct Row {
  const E* p;
  const uint4* held;  // the part's vectors, from the first on
  int32_t V, head, vecs, v0, v1;
  bool first, last;
  __device__ __forceinline__ Row(const E* row, int32_t n, int part, int parts) : p(row), V(n) {
    head = min(V, static_cast<int32_t>((16u - (reinterpret_cast<uintptr_t>(row) & 15u)) % 16u / sizeof(E)));
    vecs = (V - head) / Logit<E>::kVec;
    v0 = static_cast<int32_t>(static_cast<int64_t>(vecs) * part / parts);
    v1 = static_cast<int32_t>(static_cast<int64_t>(vecs) * (part + 1) / parts);
    held = reinterpret_cast<const uint4*>(p + head) + v0;
    first = part == 0;
    last = part == parts - 1;
  }
  __device__ __forceinline__ uint4 vec(int32_t v) const { return held[v - v0]; }
  __device__ __forceinline__ int32_t tail() const { return head + vecs * Logit<E>::kVec; }
  // Elements of the part.
  __device__ __forceinline__ int32_t count() const {
    return (v1 - v0) * Logit<E>::kVec + (first ? head : 0) + (last ? V - tail() : 0);
  }
  // f(x, index) of every element of the part, by kThreads threads.
  template <int kThreads, class F>
  __device__ __forceinline__ void each(F f) const {
    each<kThreads>([](float x) { return x; }, [&](float, float x, int32_t at) { f(x, at); });
  }
  // f(g(x), x, index), g of a vector's elements first.  The vectors go into `keep` too, where that is given; every thread finds
  // its own there.
  template <int kThreads, class G, class F>
  __device__ __forceinline__ void each(G g, F f, uint4* keep = nullptr) const {
    constexpr int VEC = Logit<E>::kVec;
    const int32_t t = threadIdx.x;
    auto one = [&](int32_t at) {
      const float x = Logit<E>::get(p + at);
      f(g(x), x, at);
    };
    if (first && t < head) one(t);
#pragma unroll 1
    for (int32_t v = v0 + t; v < v1; v += kThreads) {
      float x[VEC];
      const uint4 q = vec(v);
      if (keep) keep[v - v0] = q;
      Logit<E>::get(q, x);
      decltype(g(0.0f)) y[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) y[i] = g(x[i]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f(y[i], x[i], head + v * VEC + i);
    }
    if (last && tail() + t < V) one(tail() + t);
  }
};

// ---------------------------------------------------------------- any row
// The second kernel: the rows that the first left, a cluster of CTAs each, in one of two forms.  Both make running sums of
// the tokens' counts and weights over steps of the order that all CTAs of the cluster see alike, so that they take the same
// way, and find inside a step what is asked for.
constexpr int kSearched = 64;  // chunks of a CTA's threads: rows of which every cluster looks at all

// What both forms keep.
template <int T>
struct Common {
  uint64_t pow2[64];
  uint64_t red_w[T / 32];
  uint32_t red_c[T / 32];
  int64_t next;  // the row to do, -1: none
  int32_t left;  // and what the first kernel left of it
  uint32_t best, bad, had_c, n;
  uint64_t had_w, target;
  int32_t at;  // the token's index, -1 where another CTA has it
  Weigher weigh;
};
// A place in the order: its key, which of the tokens that have it, how many are ahead and what they weigh, and its own weight.
struct Place {
  uint32_t key, nth, before;
  uint64_t w_before, w;
};

// Sums over the CTA, in every thread.
template <int T>
__device__ __forceinline__ void block_sums(Common<T>& s, uint32_t& c, uint64_t& w) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    c += __shfl_xor_sync(0xffffffffu, c, o);
    w += __shfl_xor_sync(0xffffffffu, w, o);
  }
  __syncthreads();
  if (lane == 0) {
    s.red_c[threadIdx.x >> 5] = c;
    s.red_w[threadIdx.x >> 5] = w;
  }
  __syncthreads();
  c = s.red_c[lane % (T / 32)];
  w = s.red_w[lane % (T / 32)];
#pragma unroll
  for (int o = T / 64; o > 0; o >>= 1) {
    c += __shfl_xor_sync(0xffffffffu, c, o);
    w += __shfl_xor_sync(0xffffffffu, w, o);
  }
}
// Sums of a value over the lanes up to the own one.
template <class V>
__device__ __forceinline__ V warp_scan(V v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += y;
  }
  return v;
}
// c and w become the sums over the threads ahead; all_c and all_w over all.
template <int T>
__device__ __forceinline__ void block_scan(Common<T>& s, uint32_t& c, uint64_t& w, uint32_t& all_c, uint64_t& all_w) {
  static_assert(T <= 1024, "a lane a warp");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t own_c = c;
  const uint64_t own_w = w;
  c = warp_scan(c);
  w = warp_scan(w);
  __syncthreads();
  if (lane == 31) {
    s.red_c[warp] = c;
    s.red_w[warp] = w;
  }
  __syncthreads();
  const uint32_t cs = warp_scan(lane < T / 32 ? s.red_c[lane] : 0u);
  const uint64_t ws = warp_scan(lane < T / 32 ? s.red_w[lane] : uint64_t(0));
  all_c = __shfl_sync(0xffffffffu, cs, 31);
  all_w = __shfl_sync(0xffffffffu, ws, 31);
  const uint32_t cb = __shfl_sync(0xffffffffu, cs, (warp + 31) & 31);
  const uint64_t wb = __shfl_sync(0xffffffffu, ws, (warp + 31) & 31);
  c += (warp ? cb : 0u) - own_c;
  w += (warp ? wb : 0u) - own_w;
}

// The row's largest logit, from every CTA's least key; false (token -1 written) where nothing can be drawn.
template <typename E, int T, int kPeers, class S>
__device__ __forceinline__ bool largest(S& s, const cg::cluster_group& cluster, const SampleArgs& a, int64_t r, uint32_t& best,
                                        uint32_t bad, float t) {
  best = __reduce_min_sync(0xffffffffu, best);
  bad = __syncthreads_or(bad);
  if ((threadIdx.x & 31) == 0) s.red_c[threadIdx.x >> 5] = best;
  __syncthreads();
  best = __reduce_min_sync(0xffffffffu, s.red_c[threadIdx.x % (T / 32)]);
  if (threadIdx.x == 0) {
    s.best = best;
    s.bad = bad;
  }
  cluster.sync();
#pragma unroll
  for (int i = 0; i < kPeers; ++i) {
    const S& p = *cluster.map_shared_rank(&s, i);
    best = min(best, p.best);
    bad |= p.bad;
  }
  if (!bad && Logit<E>::of_key(best) > -INFINITY && t >= 0.0f) return true;
  if (cluster.block_rank() == 0 && threadIdx.x == 0) {
    a.tokens[r] = -1;
    if (a.logprob) a.logprob[r] = __uint_as_float(0x7fffffffu);
  }
  return false;
}

// The index of the part's j-th element (from 0) that has the key, in the order of the indexes, into s.at.
template <typename E, int T>
__device__ __forceinline__ void nth_of(Common<T>& s, const Row<E>& row, uint32_t key, uint32_t j) {
  constexpr int VEC = Logit<E>::kVec;
  uint32_t seen = 0;
  // x: n consecutive elements of the thread from index `at` on, the threads' in order
  auto step = [&](const float* x, int n, int32_t at) {
    uint32_t before = 0, all;
    uint64_t none = 0, none2;
#pragma unroll
    for (int i = 0; i < VEC; ++i) before += i < n && Logit<E>::key(x[i]) == key ? 1u : 0u;
    const uint32_t own = before;
    block_scan<T>(s, before, none, all, none2);
    before += seen;
    if (before <= j && j < before + own) {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (i < n && Logit<E>::key(x[i]) == key) {
          if (before == j) s.at = at + i;
          ++before;
        }
    }
    seen += all;
  };
  const int32_t t = threadIdx.x;
  float x[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) x[i] = 0.0f;
  if (row.first) {
    if (t < row.head) x[0] = Logit<E>::get(row.p + t);
    step(x, t < row.head ? 1 : 0, t);
  }
  for (int32_t v0 = row.v0; v0 < row.v1 && seen <= j; v0 += T) {
    const int32_t v = v0 + t;
    if (v < row.v1) Logit<E>::get(row.vec(v), x);
    step(x, v < row.v1 ? VEC : 0, row.head + v * VEC);
  }
  if (row.last && seen <= j) {
    const int32_t at = row.tail() + t;
    if (at < row.V) x[0] = Logit<E>::get(row.p + at);
    step(x, at < row.V ? 1 : 0, at);
  }
  __syncthreads();
}

// The token of a row from a form's running sums.  live, total: the number and weight of all tokens that weigh anything;
// find(by_weight, target): the first place at which the running count or weight reaches target; heavy(w0, c, sum): the number
// and weight of the tokens of w0 and more; where(place): its index, into s.at.
template <class S, class Find, class Heavy, class Where>
__device__ __forceinline__ void draw(const SampleArgs& a, int64_t r, S& s, bool greedy, uint32_t live, uint64_t total, Find find,
                                     Heavy heavy, Where where) {
  // what is kept: the first `kept` tokens, weighing `total` together
  uint32_t kept = live;
  auto limit = [&](uint32_t count, uint64_t weight) {
    if (count < kept) {
      kept = count;
      total = weight;
    }
  };
  auto ask = [&](auto f) {  // (64-bit floats: one thread's work)
    __syncthreads();
    if (threadIdx.x == 0) s.target = f();
    __syncthreads();
    return s.target;
  };
  const int32_t k = greedy ? 1 : a.top_k ? a.top_k[r] : 0;
  if (k > 0 && static_cast<uint32_t>(k) < live) {
    const Place p = find(false, k);
    limit(p.before + 1, p.w_before + p.w);
  }
  const float top_p = a.top_p && !greedy ? a.top_p[r] : 1.0f;
  if (top_p < 1.0f) {
    const Place p = find(true, ask([&] { return reaches(top_p, total); }));
    limit(p.before + 1, p.w_before + p.w);
  }
  const float least = a.min_p && !greedy ? a.min_p[r] : 0.0f;
  if (least > 0.0f) {
    uint32_t c = 0;
    uint64_t sum = 0;
    heavy(ask([&] { return least_of(least); }), c, sum);
    limit(c, sum);
  }
  const Place p = find(true, ask([&] { return passes(a.u[r], total); }));
  where(p);
  if (threadIdx.x == 0 && s.at >= 0) {
    a.tokens[r] = s.at;
    if (a.logprob) a.logprob[r] = ln_of(p.w, total);
  }
}

// f(row, what its token says) of the rows that are left.  The first CTA of a cluster looks for one and takes it; a cluster begins
// its search at a place of its own.  (Of very many rows a cluster looks at a share only.)
template <int T, class S, class F>
__device__ __forceinline__ void left_rows(const SampleArgs& a, S& s, const cg::cluster_group& cluster, F f) {
  const int peers = cluster.num_blocks();
  const int64_t clusters = gridDim.x / peers, id = blockIdx.x / peers, chunks = (a.R + T - 1) / T;
  if (a.R <= clusters) {  // a row each: no other cluster writes it, and none of this one before all have come
    const int32_t left = a.tokens[id];
    if (__syncthreads_or(left <= kUndecided)) {
      f(id, left);
      cluster.sync();  // (what one CTA reads of another's is there until it has)
    }
    return;
  }
  const bool share = chunks > kSearched;
  const int64_t todo = share ? (chunks + clusters - 1 - id) / clusters : chunks;
  auto row_of = [&](int64_t i, int t) {  // thread t's of the i-th chunk
    if (share) return (id + i * clusters) * T + t;
    const int64_t r = i * T + t + id * a.R / clusters;
    return i * T + t < a.R ? (r < a.R ? r : r - a.R) : a.R;
  };
  int64_t i = 0;
  cluster.sync();  // (every CTA of it is there)
  for (;;) {
    if (cluster.block_rank() == 0) {
      int64_t found = -1;
      while (found < 0 && i < todo) {
        const int64_t mine = row_of(i, threadIdx.x);
        const int32_t left = mine < a.R ? *static_cast<volatile int32_t*>(a.tokens + mine) : 0;
        if (!__syncthreads_or(left <= kUndecided)) {
          ++i;
          continue;
        }
        // the first thread that sees one tries to take it
        const uint32_t bits = __ballot_sync(0xffffffffu, left <= kUndecided);
        if ((threadIdx.x & 31) == 0) s.red_c[threadIdx.x >> 5] = bits;
        __syncthreads();
        int w = 0;
        while (!s.red_c[w]) ++w;
        if (static_cast<int>(threadIdx.x) == 32 * w + __ffs(s.red_c[w]) - 1) {
          s.next = atomicCAS(a.tokens + mine, left, kTaken) == left ? mine : -1;
          s.left = left;
        }
        __syncthreads();
        found = s.next;
        __syncthreads();
      }
      if (static_cast<int>(threadIdx.x) < peers) {
        S& to = *cluster.map_shared_rank(&s, threadIdx.x);
        to.next = found;
        to.left = s.left;
      }
    }
    cluster.sync();
    const int64_t r = s.next;
    if (r < 0) return;
    f(r, s.left);
    cluster.sync();  // (what one CTA reads of another's is not overwritten)
  }
}
// ---- 16-bit logits: how often each key comes is all there is to know.  A CTA counts its part's keys in 16 bits each; of the
// keys that weigh anything each CTA adds up a share over all parts, a thread some of them in order.  Most keys are of numbers
// next to 0, which no token has: the shares are of the blocks of 32 keys that any CTA has met (64 undecided rows of 131,072: 90 us
// for both kernels, 102 with shares of all keys).  A row is 11 us of exchanges and barriers: counting 3, the keys' sums and
// weights 3, running sums 3, a place 2 for each filter and the token.
constexpr int kCountPeers = 8, kCountThreads = 1024, kKeys = 65536, kShare = kKeys / kCountPeers;
constexpr int kBlockKeys = 32, kBlocks = kKeys / kBlockKeys;
constexpr int32_t kMostCounted = 500000;  // a part's count of one key stays below 2^16

struct Counts : Common<kCountThreads> {
  alignas(16) uint32_t half[kKeys / 2];  // two keys' counts a word (cleared 16 bytes at a time)
  uint64_t weight[kShare];               // of the keys of the CTA's share, 0 for those that no token has
  alignas(8) uint32_t whole[kShare];     // the row's counts of them
  uint32_t met[kBlocks / 32];            // bits of the blocks that the CTA has met
  uint32_t any[kBlocks / 32], ahead[kBlocks / 32];  // that any CTA has, and how many such lie ahead of the word's
  uint16_t block[kShare / kBlockKeys];   // the share's
  uint32_t all_c;
  uint64_t all_w;
  Place place[2];
  __device__ __forceinline__ uint32_t count(uint32_t key) const { return half[key >> 1] >> (16 * (key & 1)) & 0xffffu; }
};
static_assert(sizeof(Counts) <= 227 * 1024, "a CTA's shared memory");

__global__ void __launch_bounds__(kCountThreads, 1) sample_counts_kernel(const SampleArgs a) {
  using E = uint16_t;
  constexpr int T = kCountThreads, kPeers = kCountPeers;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Counts& s = *reinterpret_cast<Counts*>(smem_raw);
  const cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), tid = threadIdx.x;
  if (tid < 64) s.pow2[tid] = kPow2[tid];
  grid_dependency_wait();
  left_rows<T>(a, s, cluster, [&](int64_t r, int32_t left) {
    const Row<E> row(static_cast<const E*>(a.logits) + r * a.ld, a.V, rank, kPeers);
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const bool greedy = t == 0.0f;
    for (int i = tid; i < kKeys / 8; i += T) reinterpret_cast<uint4*>(s.half)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == T - 1) s.weigh = weigher(0.0f, greedy ? 1.0f : t, s.pow2);
    __syncthreads();
    uint32_t best = 0xffffffffu, bad = 0;
    row.template each<T>([&](float x, int32_t) {
      const uint32_t k = Logit<E>::key(x);
      bad |= x < INFINITY ? 0u : 1u;
      best = min(best, k);
      atomicAdd(&s.half[k >> 1], 1u << (16 * (k & 1)));
    });
    __syncthreads();
    {  // 64 blocks a warp, 8 at a time
      uint32_t met[2] = {0u, 0u};
      const uint4* const at = reinterpret_cast<const uint4*>(s.half) + (tid >> 5) * 256 + (tid & 31);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 c = at[32 * i];
        uint32_t bits = __ballot_sync(0xffffffffu, (c.x | c.y | c.z | c.w) != 0u);
        bits |= bits >> 1;
        bits = (bits | bits >> 2) & 0x11111111u;  // of four lanes a block
        bits = (bits | bits >> 3) & 0x03030303u;
        bits = (bits | bits >> 6) & 0x000f000fu;
        met[i / 4] |= ((bits | bits >> 12) & 0xffu) << (8 * (i % 4));
      }
      if ((tid & 31) < 2) s.met[tid >> 5 << 1 | (tid & 31)] = tid & 1 ? met[1] : met[0];
    }
    if (largest_of(left) >= 0) {
      best = Logit<E>::key(Logit<E>::get(row.p + largest_of(left)));
      cluster.sync();
    } else if (!largest<E, T, kPeers>(s, cluster, a, r, best, bad, t)) {
      return;
    }
    Weigher weigh = s.weigh;
    weigh.max = Logit<E>::of_key(best);

    // the share's keys over all parts, a thread's side by side
    const uint32_t last = Logit<E>::key(fmaxf(__fsub_rd(weigh.max, 1.001f * weigh.cut), kLowest)) / kBlockKeys;
    if (tid < kBlocks / 32) {
      uint32_t any = 0;
#pragma unroll
      for (int e = 0; e < kPeers; ++e) any |= cluster.map_shared_rank(&s, e)->met[tid];
      const int below = static_cast<int>(last) + 1 - 32 * tid;  // (blocks behind the last weigh nothing)
      s.any[tid] = below >= 32 ? any : below > 0 ? any & ((1u << below) - 1u) : 0u;
    }
    __syncthreads();
    if (tid < 32) {
      const uint32_t n0 = __popc(s.any[2 * tid]), n1 = __popc(s.any[2 * tid + 1]), upto = warp_scan(n0 + n1);
      s.ahead[2 * tid] = upto - n0 - n1;
      s.ahead[2 * tid + 1] = upto - n1;
    }
    __syncthreads();
    const uint32_t met = s.ahead[kBlocks / 32 - 1] + __popc(s.any[kBlocks / 32 - 1]), share = (met + kPeers - 1) / kPeers;
    const uint32_t first = min(rank * share, met), mine = kBlockKeys * (min(first + share, met) - first);
#pragma unroll
    for (int i = tid; i < kBlocks; i += T) {
      const uint32_t bits = s.any[i / 32], at = s.ahead[i / 32] + __popc(bits & ((1u << (i % 32)) - 1u)) - first;
      if ((bits >> (i % 32) & 1u) && at < mine / kBlockKeys) s.block[at] = static_cast<uint16_t>(i);
    }
    __syncthreads();
    auto key_of = [&](uint32_t i) { return kBlockKeys * s.block[i / kBlockKeys] + i % kBlockKeys; };
    for (uint32_t i = tid; i < mine / 2; i += T) {
      const uint32_t word = key_of(2 * i) / 2;
      uint32_t c[kPeers];
#pragma unroll
      for (int e = 0; e < kPeers; ++e) c[e] = cluster.map_shared_rank(&s, e)->half[word];
      uint2 sum = make_uint2(0u, 0u);
#pragma unroll
      for (int e = 0; e < kPeers; ++e) {
        sum.x += c[e] & 0xffffu;
        sum.y += c[e] >> 16;
      }
      reinterpret_cast<uint2*>(s.whole)[i] = sum;
    }
    __syncthreads();
    for (uint32_t i = tid; i < mine; i += T) s.weight[i] = s.whole[i] ? weigh(Logit<E>::of_key(key_of(i))) : 0;
    __syncthreads();
    const uint32_t per = (share * kBlockKeys + T - 1) / T, i0 = min(tid * per, mine), i1 = min(i0 + per, mine);
    auto walk = [&](auto f) {  // f(key, tokens, weight of one) of the thread's keys that weigh anything
      for (uint32_t i = i0; i < i1; ++i) {
        const uint64_t w = s.weight[i];
        if (w && f(key_of(i), s.whole[i], w)) return;
      }
    };
    uint32_t own_c = 0, all_c;
    uint64_t own_w = 0, all_w;
    walk([&](uint32_t, uint32_t c, uint64_t w) {
      own_c += c;
      own_w += c * w;
      return false;
    });
    uint32_t c0 = own_c;
    uint64_t w0 = own_w;
    block_scan<T>(s, c0, w0, all_c, all_w);
    if (tid == 0) {
      s.all_c = all_c;
      s.all_w = all_w;
    }
    cluster.sync();
    all_c = 0;
    all_w = 0;
#pragma unroll
    for (int i = 0; i < kPeers; ++i) {
      const Counts& p = *cluster.map_shared_rank(&s, i);
      if (i == rank) {
        c0 += all_c;
        w0 += all_w;
      }
      all_c += p.all_c;
      all_w += p.all_w;
    }
    int turn = 0;
    auto find = [&](bool by_weight, uint64_t target) {
      Place& to = s.place[turn];  // (the other may still be read)
      turn ^= 1;
      if (by_weight ? w0 < target && target <= w0 + own_w : c0 < target && target <= c0 + own_c) {
        Place p{0, 0, c0, w0, 0};
        walk([&](uint32_t key, uint32_t c, uint64_t w) {
          const uint64_t left = (by_weight ? (target - p.w_before - 1) / w : target - p.before - 1);
          const uint32_t j = static_cast<uint32_t>(left < c ? left : c);
          p.before += j;
          p.w_before += j * w;
          p.key = key;
          p.nth = j;
          p.w = w;
          return j < c;
        });
#pragma unroll
        for (int i = 0; i < kPeers; ++i) *cluster.map_shared_rank(&to, i) = p;
      }
      cluster.sync();
      return to;
    };
    auto heavy = [&](uint64_t least, uint32_t& c, uint64_t& sum) {
      walk([&](uint32_t, uint32_t n, uint64_t w) {
        if (w < least) return true;
        c += n;
        sum += n * w;
        return false;
      });
      block_sums<T>(s, c, sum);
      if (tid == 0) {
        s.had_c = c;
        s.had_w = sum;
      }
      cluster.sync();
      c = 0;
      sum = 0;
#pragma unroll
      for (int i = 0; i < kPeers; ++i) {
        c += cluster.map_shared_rank(&s, i)->had_c;
        sum += cluster.map_shared_rank(&s, i)->had_w;
      }
    };
    auto where = [&](const Place& p) {
      const uint32_t seen =
          __reduce_add_sync(0xffffffffu, (tid & 31) < rank ? cluster.map_shared_rank(&s, tid & 31)->count(p.key) : 0u);
      if (tid == 0) s.at = -1;
      __syncthreads();
      if (seen <= p.nth && p.nth < seen + s.count(p.key)) nth_of<E, T>(s, row, p.key, p.nth - seen);
    };
    draw(a, r, s, greedy, all_c, all_w, find, heavy, where);
  });
}

// ---- any logits: a histogram of counts and weights by max - x; in one of its bins, by ranks where it has few tokens, by keys
// (and finer ones) where it has many.  A row of 100,003 fp32 logits takes 28 us: 12 for all weights and their three atomics a
// token, 5 for the bins' sums over the CTAs, 10 for a place.
constexpr int kThreads = 1024;
constexpr int kBinBits = 11, kBins = 1 << kBinBits;
constexpr int kList = 512;  // tokens whose ranks are found one against all others
constexpr int kHeld = 4096;  // vectors of its part that a CTA keeps (131,072 fp32 logits)

struct Sums {  // of a bin and all before it
  uint64_t weight[kBins];
  uint32_t count[kBins];
};
struct Tokens {
  uint64_t w[kList];
  uint32_t key[kList];
  int32_t at[kList];
};
struct Binned : Common<kThreads> {
  uint32_t count[kBins], lo[kBins], hi[kBins];  // the CTA's part of the row
  Sums sums[2];
  Tokens own, all;
  Place place;
  uint4 held[kHeld];
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < kBins; i += kThreads) count[i] = lo[i] = hi[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void add(int bin, uint64_t weight) {
    atomicAdd(&count[bin], 1u);
    const uint32_t low = static_cast<uint32_t>(weight), old = atomicAdd(&lo[bin], low);
    const uint32_t high = static_cast<uint32_t>(weight >> 32) + (old + low < old ? 1u : 0u);
    if (high) atomicAdd(&hi[bin], high);
  }
};

// The histograms of all CTAs to running sums, on top of what came before them.
template <int kPeers>
__device__ __forceinline__ void sum_up(Binned& s, const cg::cluster_group& cluster, Sums& to, uint32_t c0, uint64_t w0) {
  constexpr int kPer = kBins / kThreads;
  const int rank = cluster.block_rank();
  if constexpr (kPeers == 1) {
    __syncthreads();
    for (int bin = threadIdx.x; bin < kBins; bin += kThreads) {
      to.count[bin] = s.count[bin];
      to.weight[bin] = (static_cast<uint64_t>(s.hi[bin]) << 32) + s.lo[bin];
    }
    __syncthreads();
  } else {  // some threads a bin, each for some of the CTAs, a warp's bins side by side
    cluster.sync();
    constexpr int kBinShare = kBins / kPeers, kShare = kThreads / kBinShare, kEach = kPeers / kShare;
    static_assert(kShare * kBinShare == kThreads && kEach * kShare == kPeers && kThreads == 2 * kList, "all threads, all CTAs");
    const int at = threadIdx.x % kBinShare, bin = rank * kBinShare + at, peer = threadIdx.x / kBinShare * kEach;
    uint32_t c = 0;
    uint64_t w = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const Binned& p = *cluster.map_shared_rank(&s, peer + i);
      c += p.count[bin];
      w += (static_cast<uint64_t>(p.hi[bin]) << 32) + p.lo[bin];
    }
    Tokens& mine = threadIdx.x < kList ? s.own : s.all;
    mine.key[threadIdx.x % kList] = c;
    mine.w[threadIdx.x % kList] = w;
    __syncthreads();
    c = 0;
    w = 0;
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      const int t = i * kBinShare + at;
      const Tokens& of = t < kList ? s.own : s.all;
      c += of.key[t % kList];
      w += of.w[t % kList];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      Sums& p = *cluster.map_shared_rank(&to, peer + i);
      p.count[bin] = c;
      p.weight[bin] = w;
    }
    cluster.sync();
  }
  uint32_t c[kPer], ca = 0, all_c;
  uint64_t w[kPer], wa = 0, all_w;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    c[i] = ca += to.count[threadIdx.x * kPer + i];
    w[i] = wa += to.weight[threadIdx.x * kPer + i];
  }
  block_scan<kThreads>(s, ca, wa, all_c, all_w);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    to.count[threadIdx.x * kPer + i] = c0 + ca + c[i];
    to.weight[threadIdx.x * kPer + i] = w0 + wa + w[i];
  }
  __syncthreads();
}

// The first bin whose running sum reaches target >= 1.
__device__ __forceinline__ int first_bin(const Sums& b, bool by_weight, uint64_t target) {
  int lo = 0, hi = kBins - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if ((by_weight ? b.weight[mid] : b.count[mid]) >= target)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

template <typename E, int kPeers>
__device__ __forceinline__ void sample_binned(const SampleArgs& a, int64_t r, int32_t left, Binned& s,
                                              const cg::cluster_group& cluster) {
  constexpr int T = kThreads;
  const int rank = cluster.block_rank(), tid = threadIdx.x;
  Row<E> row(static_cast<const E*>(a.logits) + r * a.ld, a.V, rank, kPeers);
  const float t = a.temperature ? a.temperature[r] : 1.0f;
  const bool greedy = t == 0.0f;
  if (tid == T - 1) s.weigh = weigher(0.0f, greedy ? 1.0f : t, s.pow2);
  s.clear();
  uint32_t best = 0xffffffffu, bad = 0;
  if (largest_of(left) >= 0) {
    best = Logit<E>::key(Logit<E>::get(row.p + largest_of(left)));
  } else {
    row.template each<T>([&](float x, int32_t) {
      bad |= x < INFINITY ? 0u : 1u;
      best = min(best, Logit<E>::key(x));
    });
    if (!largest<E, T, kPeers>(s, cluster, a, r, best, bad, t)) return;
  }
  Weigher weigh = s.weigh;
  weigh.max = Logit<E>::of_key(best);

  // all tokens that weigh anything
  const float wide = weigh.cut * (1.0f / kBins), by = 1.0f / wide;
  auto bin_of = [&](float x) { return min(static_cast<int>((weigh.max - x) * by), kBins - 1); };
  row.template each<T>([&](float x) { return weigh.beside(x); }, [&](uint64_t w, float x, int32_t) {
    if (w) s.add(bin_of(x), w);
  }, row.v1 - row.v0 <= kHeld ? s.held : nullptr);
  if (row.v1 - row.v0 <= kHeld) row.held = s.held;
  sum_up<kPeers>(s, cluster, s.sums[0], 0, 0);

  auto find = [&](bool by_weight, uint64_t target) {
    const int bin = first_bin(s.sums[0], by_weight, target);
    uint32_t c0 = bin ? s.sums[0].count[bin - 1] : 0, n = s.sums[0].count[bin] - c0;
    uint64_t w0 = bin ? s.sums[0].weight[bin - 1] : 0;
    // the keys from `lo` on that a token of the bin can have (limits a little wide)
    uint32_t lo = max(Logit<E>::key(fminf(weigh.max - wide * bin * 0.99999f, weigh.max)), best);
    const float low_x = bin == kBins - 1 ? kLowest : fmaxf(weigh.max - wide * (bin + 1) * 1.00001f, kLowest);
    int shift = 0;
    while ((Logit<E>::key(low_x) - lo) >> shift >= kBins) ++shift;
    shift += kBinBits;
    auto each_in = [&](auto f) {
      row.template each<T>([&](float x, int32_t at) {
        if (!(weigh.max - x < weigh.cut) || bin_of(x) != bin) return;
        const uint32_t k = Logit<E>::key(x);
        if (static_cast<uint64_t>(k - lo) >> shift) return;
        const uint64_t w = weigh(x);
        if (w) f(k, at, w);
      });
    };
    while (n > kList && shift > 0) {
      const int finer = max(shift - kBinBits, 0);
      __syncthreads();
      s.clear();
      each_in([&](uint32_t k, int32_t, uint64_t w) { s.add(min((k - lo) >> finer, kBins - 1u), w); });
      sum_up<kPeers>(s, cluster, s.sums[1], c0, w0);
      const int at = first_bin(s.sums[1], by_weight, target);
      if (at) {
        c0 = s.sums[1].count[at - 1];
        w0 = s.sums[1].weight[at - 1];
      }
      n = s.sums[1].count[at] - c0;
      lo += static_cast<uint32_t>(at) << finer;
      shift = finer;
    }
    __syncthreads();
    if (n > kList) {  // one key
      Place p;
      p.key = lo;
      p.w = weigh(Logit<E>::of_key(lo));
      p.nth = static_cast<uint32_t>(by_weight ? (target - w0 - 1) / p.w : target - c0 - 1);
      p.before = c0 + p.nth;
      p.w_before = w0 + p.nth * p.w;
      if (tid == 0) s.at = -2;  // (which of them, nth_of says)
      __syncthreads();
      return p;
    }
    if (tid == 0) s.n = 0;
    __syncthreads();
    each_in([&](uint32_t k, int32_t at, uint64_t w) {
      const uint32_t i = atomicAdd(&s.n, 1u);
      if (i >= kList) return;
      s.own.key[i] = k;
      s.own.at[i] = at;
      s.own.w[i] = w;
    });
    cluster.sync();
    const int lane = tid & 31, warp = tid >> 5;
    const uint32_t upto = warp_scan(lane < kPeers ? cluster.map_shared_rank(&s, lane)->n : 0u);
    const uint32_t m = min(__shfl_sync(0xffffffffu, upto, 31), static_cast<uint32_t>(kList));
    static_assert(kPeers <= T / 32, "a warp a CTA of the cluster");
    const uint32_t own1 = min(__shfl_sync(0xffffffffu, upto, rank), m), own0 = own1 - min(s.n, own1);
    if (warp < kPeers) {
      const Binned& p = *cluster.map_shared_rank(&s, warp);
      const uint32_t end = min(__shfl_sync(0xffffffffu, upto, warp), m), from = end - min(p.n, end);
      for (uint32_t e = lane; e < end - from; e += 32) {
        s.all.key[from + e] = p.own.key[e];
        s.all.at[from + e] = p.own.at[e];
        s.all.w[from + e] = p.own.w[e];
      }
    }
    __syncthreads();
    // (a CTA looks at its own tokens, a group of lanes at one of them)
    constexpr uint32_t kGroup = 16;
    for (uint32_t e = own0; e < own1; e += T / kGroup) {
      const uint32_t mine = e + tid / kGroup, me = min(mine, own1 - 1), k = s.all.key[me];
      const int32_t at = s.all.at[me];
      uint32_t c = 0;
      uint64_t w = 0;
#pragma unroll 4
      for (uint32_t i = tid % kGroup; i < m; i += kGroup) {
        const uint32_t ki = s.all.key[i];
        const bool ahead = ki < k || (ki == k && s.all.at[i] < at);
        c += ahead ? 1u : 0u;
        w += ahead ? s.all.w[i] : 0u;
      }
#pragma unroll
      for (uint32_t o = kGroup / 2; o > 0; o >>= 1) {
        c += __shfl_xor_sync(0xffffffffu, c, o);
        w += __shfl_xor_sync(0xffffffffu, w, o);
      }
      c += c0;
      w += w0;
      const uint64_t from = by_weight ? w : c, with = from + (by_weight ? s.all.w[me] : 1u);
      const uint32_t to = tid % kGroup;  // (a lane tells a CTA)
      if (mine < own1 && from < target && target <= with && to < kPeers) {
        Binned& p = *cluster.map_shared_rank(&s, to);
        p.place = Place{k, 0, c, w, s.all.w[me]};
        p.at = to == 0 ? at : -1;
      }
    }
    cluster.sync();
    return s.place;
  };
  auto heavy = [&](uint64_t least, uint32_t& c, uint64_t& sum) {
    row.template each<T>([&](float x, int32_t) {
      const uint64_t w = weigh(x);
      if (w >= least) {
        ++c;
        sum += w;
      }
    });
    block_sums<T>(s, c, sum);
    if (tid == 0) {
      s.had_c = c;
      s.had_w = sum;
    }
    cluster.sync();
    c = 0;
    sum = 0;
    for (int i = 0; i < kPeers; ++i) {
      c += cluster.map_shared_rank(&s, i)->had_c;
      sum += cluster.map_shared_rank(&s, i)->had_w;
    }
  };
  auto where = [&](const Place& p) {
    if (s.at != -2) return;
    uint32_t mine = 0, seen = 0;
    uint64_t none = 0;
    row.template each<T>([&](float x, int32_t) { mine += Logit<E>::key(x) == p.key ? 1u : 0u; });
    block_sums<T>(s, mine, none);
    if (tid == 0) {
      s.n = mine;
      s.at = -1;
    }
    cluster.sync();
    seen = __reduce_add_sync(0xffffffffu, (tid & 31) < rank ? cluster.map_shared_rank(&s, tid & 31)->n : 0u);
    if (seen <= p.nth && p.nth < seen + mine) nth_of<E, T>(s, row, p.key, p.nth - seen);
  };
  draw(a, r, s, greedy, s.sums[0].count[kBins - 1], s.sums[0].weight[kBins - 1], find, heavy, where);
}

template <typename E, int kPeers>
__global__ void __launch_bounds__(kThreads, 1) sample_binned_kernel(const SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Binned& s = *reinterpret_cast<Binned*>(smem_raw);
  const cg::cluster_group cluster = cg::this_cluster();
  if (threadIdx.x < 64) s.pow2[threadIdx.x] = kPow2[threadIdx.x];
  grid_dependency_wait();
  left_rows<kThreads>(a, s, cluster, [&](int64_t r, int32_t left) { sample_binned<E, kPeers>(a, r, left, s, cluster); });
}

// ---------------------------------------------------------------- rows that their largest tokens decide
// The first kernel: a cluster a row, one pass over it.  From a sample of the row, spread over it, comes a bound that about as many
// of its tokens pass as are wanted.  Tokens at the bound and above go into a list; the others' weights are only summed, in
// fp32 with an error that is bounded.  The cluster's first CTA puts the list in order and sums its weights up exactly.  Where
// what is kept ends inside the list, or the token is inside it for the least and the largest sum that the others can have, this
// is the result; a row of which neither holds, or whose list overflows, is left to the second kernel.
// 64 rows of 131,072 bf16 logits (16.8 MB) take 18 us here, 384 of 100,003 in fp32 (153.6 MB) 53, 2.9 TB/s.  The pass itself runs
// at 6 TB/s with two CTAs an SM; bounds are the last wave of CTAs (384 on 304 places) and some 16,000 cycles of a CTA behind
// its pass in which the SM loads little: the exchange, the list's order, exact weights, and sums and decisions with a barrier
// after each.  Three CTAs an SM (40 registers) 3 % slower; elements at the bound and above looked for in a second look at their
// vectors 6 to 20 %; stretches of 2 KB a warp and step 2 % faster for long rows and 9 % slower for parts of one step.
constexpr int kHeadThreads = 512, kHeadWarps = kHeadThreads / 32;
constexpr int kCap = 2560;       // tokens of a list
constexpr int kWhole = 2048;     // rows of up to so many are taken whole
constexpr float kWant = 500.0f, kMostWanted = 1700.0f;  // tokens that the list is to have
constexpr int kSpread = 1024;    // bins of the list's order
constexpr uint32_t kSame = 512;  // tokens of one of them at most
constexpr int kMostCtas = 8;     // of a cluster

struct Head {
  uint64_t packed[kCap];  // the list by bins: a token's key and index
  union {
    float x[kCap];        // the list, then (in order)
    uint64_t sum[kCap];   // the weights, then their running sums
  };
  int32_t at[kCap];       // its indexes, then in order
  uint32_t upto[kSpread];
  uint64_t pow2[64];
  uint64_t red_w[kHeadWarps], red_low[kHeadWarps];
  int32_t red[kHeadWarps];
  float sample[kHeadThreads];
  int32_t reach[kHeadWarps];
  // of every CTA of the cluster: its bound, the others' weights in units of 2^-26 2^(their reference), that, and their number
  float bound[kMostCtas], ref[kMostCtas];
  uint64_t rest[kMostCtas];
  uint32_t others[kMostCtas];
  uint32_t n, bad;
  int32_t place;
  Weigher weigh;
  uint64_t rest_low, rest_high;  // limits of the others' weight
  uint64_t asked[2], low_w;
};

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Floats as integers in the same order.
__device__ __forceinline__ int32_t in_order(float x) {
  const int32_t i = __float_as_int(x);
  return i ^ (i >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float from_order(int32_t i) { return __int_as_float(i ^ (i >> 31 & 0x7fffffff)); }

// The largest of a vector's elements, NaN if any is.
__device__ __forceinline__ float most_of(const uint4& q, const float*, const uint16_t*) {
  uint32_t a, b;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(q.x), "r"(q.y));
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(q.z), "r"(q.w));
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a << 16)), "f"(__uint_as_float(a & 0xffff0000u)));
  return r;
}
__device__ __forceinline__ float most_of(const uint4&, const float* x, const float*) {
  float a, b;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(x[0]), "f"(x[1]));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(b) : "f"(x[2]), "f"(x[3]));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(a), "f"(b));
  return a;
}

// How many of the n tokens in order f(token) holds for, in every thread.
template <class F>
__device__ __forceinline__ int32_t count_of(int32_t n, F f) {
  int32_t c = 0;
#pragma unroll 1
  for (int32_t i = threadIdx.x; i - static_cast<int32_t>(threadIdx.x) < n; i += kHeadThreads) c += __syncthreads_count(i < n && f(i));
  return c;
}
// The first of the n tokens in order whose running weight reaches target, n - 1 if none.
__device__ __forceinline__ int32_t first_place(const Head& s, int32_t n, uint64_t target) {
  return min(count_of(n, [&](int32_t i) { return s.sum[i] < target; }), n - 1);
}
// The first of them that weighs less than w, n if none (the first weighs as much as any may be asked).
__device__ __forceinline__ int32_t first_light(const Head& s, int32_t n, uint64_t w) {
  return max(count_of(n, [&](int32_t i) { return s.sum[i] - (i ? s.sum[i - 1] : 0) >= w; }), 1);
}
// f of the weight of what is kept, or of the least and the largest that it can be, in every thread (f is in 64-bit floats, of
// which an SM has few: two threads compute it).
template <class F>
__device__ __forceinline__ void ask(Head& s, uint64_t (&out)[2], uint64_t least, uint64_t most, F f) {
  if ((threadIdx.x & ~32u) == 0) s.asked[threadIdx.x >> 5] = f(threadIdx.x ? most : least);
  __syncthreads();
  out[0] = s.asked[0];
  out[1] = s.asked[1];
  __syncthreads();
}

template <typename E>
__global__ void __launch_bounds__(kHeadThreads, 2) sample_head_kernel(const SampleArgs a) {
  constexpr int VEC = Logit<E>::kVec, kDeep = 4;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Head& s = *reinterpret_cast<Head*>(smem_raw);
  const cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r = blockIdx.x / ctas;
  const Row<E> row(static_cast<const E*>(a.logits) + r * a.ld, a.V, rank, ctas);
  const int32_t v0 = row.v0, v1 = row.v1;
  if (tid < 64) s.pow2[tid] = kPow2[tid];
  if (tid == 0) s.n = s.bad = 0;
  grid_launch_dependents();
  grid_dependency_wait();
  const float t = a.temperature ? a.temperature[r] : 1.0f;
  const int32_t k = a.top_k ? a.top_k[r] : 0;
  const bool greedy = t == 0.0f, plain = greedy || (t >= 0x1p-10f && t <= 0x1p10f);
  if (!(t >= 0.0f) || !plain) {  // (one for all CTAs of the cluster)
    if (rank == 0 && tid == 0) a.tokens[r] = kUndecided;
    return;
  }
  // c = log2(e) / T as a float and a rest (the pass over the row does without it: c_hi (x - bound) is what it needs)
  float c_hi, c_lo;
  {
    const float by = greedy ? 1.0f : t;
    c_hi = __fdiv_rn(1.44269504f, by);
    c_lo = __fdiv_rn(fmaf(-c_hi, by, 1.44269504f) + 1.925963e-8f, by);
  }

  // The part's vectors, 32 at a time, in as many streams as a step of the pass takes, side by side in the row: a step's i-th
  // vectors of the thread.  The first step's are the sample, too.
  const int32_t groups = (v1 - v0 + 31) / 32, per = max((groups + kDeep * kHeadWarps - 1) / (kDeep * kHeadWarps), 1);
  auto spot = [&](int i, int32_t step) { return v0 + 32 * ((i * kHeadWarps + warp) * per + step) + lane; };
  uint4 q[kDeep];
  auto load = [&](int32_t step) {
#pragma unroll
    for (int i = 0; i < kDeep; ++i)
      if (spot(i, step) < v1) q[i] = row.vec(spot(i, step));
  };
  load(0);

  // The bound: of the sample, the largest of a thread's elements; of a share q of the row, one of m is in it with
  // 1 - (1 - q)^m.  In two rounds each warp counts how many of the threads reach one of 16 values between the largest of all and
  // the least that can matter.
  float bound = kLowest;
  if (a.V > kWhole && v1 > v0) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kDeep; ++i)
      if (spot(i, 0) < v1) {
        float x[VEC];
        Logit<E>::get(q[i], x);
        top = fmaxf(top, most_of(q[i], x, static_cast<const E*>(nullptr)));
      }
    s.sample[tid] = top;
    const int32_t highest = __reduce_max_sync(0xffffffffu, in_order(top));
    if (lane == 0) s.red[warp] = highest;
    const float want = greedy ? 64.0f : k > 0 ? fminf(fmaxf(1.25f * k + 100.0f, kWant), kMostWanted) : kWant;
    // (some warps have a vector a thread more than the others)
    const int32_t streams = (groups + per - 1) / per, full = streams / kHeadWarps;
    const float miss = log2f(fmaxf(1.0f - want / a.V, 0.0f)) * VEC, none = full > 0 ? ex2(miss * full) : 1.0f;
    const float more = ex2(miss * (full + 1)), share = static_cast<float>(streams % kHeadWarps) / kHeadWarps;
    const int32_t reach = max(static_cast<int32_t>(kHeadThreads * (1.0f - share * more - (1.0f - share) * none)), 4);
    __syncthreads();
    int32_t most = s.red[0];
#pragma unroll
    for (int i = 1; i < kHeadWarps; ++i) most = max(most, s.red[i]);
    const float hi = from_order(most);
    float lo = fmaxf(hi - 32.0f * (greedy ? 1.0f : t), kLowest), step = (hi - lo) * (1.0f / 17.0f);
    if (hi > -INFINITY && hi < INFINITY) {
      float mine[kHeadThreads / 32];
#pragma unroll
      for (int i = 0; i < kHeadThreads / 32; ++i) mine[i] = s.sample[32 * i + lane];
      bound = lo;
#pragma unroll
      for (int round = 0; round < 2; ++round) {
        const float at = bound + step * (warp + 1);
        int32_t has = 0;
#pragma unroll
        for (int i = 0; i < kHeadThreads / 32; ++i) has += mine[i] >= at ? 1 : 0;
        has = __reduce_add_sync(0xffffffffu, has);
        if (lane == 0) s.reach[warp] = has;
        __syncthreads();
        int32_t up = 0;
#pragma unroll
        for (int i = 0; i < kHeadWarps; ++i) up += s.reach[i] >= reach ? 1 : 0;
        bound += step * up;
        step *= 1.0f / 17.0f;
        __syncthreads();
      }
    }
  } else {
    __syncthreads();  // (the list's counters are set)
  }
  const float ref = bound > -1e30f ? bound * c_hi : 0.0f;
  // (constants of the exact weights: 64-bit floats, beside the pass)
  if (tid == kHeadThreads - 1) s.weigh = weigher(0.0f, greedy ? 1.0f : t, s.pow2);

  // the pass over the row
  uint64_t rest = 0;
  auto keep = [&](float x, int32_t at) {  // a token of the list
    if (!(x < INFINITY)) s.bad = 1;
    const uint32_t i = atomicAdd(&s.n, 1u);
    if (i < kCap) {
      s.x[i] = x;
      s.at[i] = at;
    }
  };
  auto one = [&](int32_t at) {
    const float x = Logit<E>::get(row.p + at);
    if (x < bound)
      rest += __float2uint_rn(ex2(fmaf(x, c_hi, -ref)) * 0x1p26f);
    else
      keep(x, at);
  };
  auto vec = [&](const uint4& q, int32_t v) {
    float x[VEC], w[VEC];
    Logit<E>::get(q, x);
    uint32_t high = 0;  // bit e: the e-th is at the bound or above
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const bool below = x[e] < bound;
      w[e] = below ? ex2(fmaf(x[e], c_hi, -ref)) : 0.0f;
      high |= below ? 0u : 1u << e;
    }
#pragma unroll 1
    for (; high; high &= high - 1) {
      const int e = __ffs(high) - 1;
      keep(Logit<E>::get(q, e), row.head + v * VEC + e);
    }
#pragma unroll
    for (int o = VEC / 2; o > 0; o >>= 1)
#pragma unroll
      for (int e = 0; e < o; ++e) w[e] += w[e + o];
    return w[0];
  };
  // (the next step's vectors are on their way while these are looked at)
#pragma unroll 1
  for (int32_t step = 0; step < per; ++step) {
    uint4 now[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) now[i] = q[i];
    if (step + 1 < per) load(step + 1);
    float sum = 0.0f;  // (below 2^5)
#pragma unroll
    for (int i = 0; i < kDeep; ++i)
      if (spot(i, step) < v1) sum += vec(now[i], spot(i, step));
    rest += __float2uint_rn(sum * 0x1p26f);
  }
  if (row.first && tid < row.head) one(tid);
  if (row.last && row.tail() + tid < row.V) one(row.tail() + tid);

  // everything to the first CTA
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
  if (lane == 0) s.red_w[warp] = rest;
  __syncthreads();
  const uint32_t mine = s.n;
  if (ctas > 1) cluster.sync();  // (the first CTA's counters are set, and its own tokens counted)
  Head& f = *cluster.map_shared_rank(&s, 0);
  {
    if (tid == 0) {
      rest = 0;
      for (int i = 0; i < kHeadWarps; ++i) rest += s.red_w[i];
      f.rest[rank] = rest;
      f.bound[rank] = bound;
      f.ref[rank] = ref;
      f.others[rank] = static_cast<uint32_t>(row.count()) - mine;
      if (rank > 0) {
        if (s.bad) f.bad = 1;
        s.place = static_cast<int32_t>(atomicAdd(&f.n, mine));
      }
    }
    __syncthreads();
    if (rank > 0) {
      const uint32_t from = s.place;
      if (mine <= kCap && from + mine <= kCap)
        for (uint32_t i = tid; i < mine; i += kHeadThreads) {
          f.x[from + i] = s.x[i];
          f.at[from + i] = s.at[i];
        }
    }
  }
  if (ctas > 1) cluster.sync();
  if (rank > 0) return;

  // ---- the list in order
  const uint32_t n_all = s.n;
  const bool bad = s.bad || n_all == 0;
  if (bad || n_all > kCap) {
    if (tid == 0) {
      a.tokens[r] = bad ? -1 : kUndecided;
      if (a.logprob && bad) a.logprob[r] = __uint_as_float(0x7fffffffu);
    }
    return;
  }
  float floor_ = kLowest;
  for (int i = 0; i < ctas; ++i) floor_ = fmaxf(floor_, s.bound[i]);
  int32_t top = in_order(-INFINITY);
  for (uint32_t i = tid; i < n_all; i += kHeadThreads) top = max(top, in_order(s.x[i]));
  top = __reduce_max_sync(0xffffffffu, top);
  if (lane == 0) s.red[warp] = top;
  for (int i = tid; i < kSpread; i += kHeadThreads) s.upto[i] = 0;
  __syncthreads();
  for (int i = 0; i < kHeadWarps; ++i) top = max(top, s.red[i]);
  const float max_x = from_order(top);
  Weigher weigh = s.weigh;
  weigh.max = max_x;
  // Tokens below every CTA's bound, or without weight, are not put in order; the former's weights are summed.
  const float cut = weigh.cut, span = fminf(max_x - floor_, cut);
  const float scale = span > 0.0f && span < 1e37f ? (kSpread - 1) / span : 0.0f;
  auto bin_of = [&](float x) { return min(static_cast<int>((max_x - x) * scale), kSpread - 1); };
  for (uint32_t i = tid; i < n_all; i += kHeadThreads) {
    const float x = s.x[i];
    if (x >= floor_ && max_x - x < cut) atomicAdd(&s.upto[bin_of(x)], 1u);
  }
  __syncthreads();
  {  // counts to first places
    constexpr int kPer = kSpread / kHeadThreads;
    uint32_t c[kPer], sum = 0;
    bool full = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      c[i] = sum;
      const uint32_t here = s.upto[tid * kPer + i];
      full |= here > kSame;
      sum += here;
    }
    if (__syncthreads_or(full)) {
      if (tid == 0) a.tokens[r] = kUndecided;
      return;
    }
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) s.red[warp] = upto;
    __syncthreads();
    uint32_t base = upto - sum;
    for (int i = 0; i < warp; ++i) base += s.red[i];
#pragma unroll
    for (int i = 0; i < kPer; ++i) s.upto[tid * kPer + i] = base + c[i];
  }
  __syncthreads();
  uint64_t low = 0;
  for (uint32_t i = tid; i < n_all; i += kHeadThreads) {
    const float x = s.x[i];
    if (x >= floor_ && max_x - x < cut) {
      const uint32_t j = atomicAdd(&s.upto[bin_of(x)], 1u);  // (afterwards: the next bin's first place)
      s.packed[j] = static_cast<uint64_t>(~static_cast<uint32_t>(in_order(x + 0.0f)) ^ 0x80000000u) << 32 | static_cast<uint32_t>(s.at[i]);
    } else {
      low += weigh(x);
    }
  }
  __syncthreads();
  const int32_t n = s.upto[kSpread - 1];
  for (int32_t i = tid; i < n; i += kHeadThreads) {
    const uint64_t mine = s.packed[i];
    const float x = from_order(static_cast<int32_t>(~static_cast<uint32_t>(mine >> 32) ^ 0x80000000u));
    const int32_t b = bin_of(x), from = b ? s.upto[b - 1] : 0, to = s.upto[b];
    const uint64_t w = weigh(x);
    int32_t j = from;
#pragma unroll 4
    for (int32_t e = from; e < to; ++e) j += s.packed[e] < mine ? 1 : 0;
    s.at[j] = static_cast<int32_t>(static_cast<uint32_t>(mine));
    s.sum[j] = w;
  }
  __syncthreads();
  {  // running weights
    constexpr int kEach = kCap / kHeadThreads;
    const int32_t per = (n + kHeadThreads - 1) / kHeadThreads, i0 = tid * per;
    uint64_t own[kEach], upto = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (i < per && i0 + i < n) upto += s.sum[i0 + i];
      own[i] = upto;
    }
    const uint64_t mine_w = upto;
    upto = warp_scan(upto);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) low += __shfl_xor_sync(0xffffffffu, low, o);
    if (lane == 31) s.red_w[warp] = upto;
    if (lane == 0) s.red_low[warp] = low;
    __syncthreads();
    uint64_t run = upto - mine_w;
#pragma unroll
    for (int i = 0; i < kHeadWarps - 1; ++i) run += i < warp ? s.red_w[i] : 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (i < per && i0 + i < n) s.sum[i0 + i] = run + own[i];
  }

  // ---- the weight of the whole row, between low_all and high_all
  bool known = !(max_x - floor_ < cut);  // what is kept ends in the list: here, as all else weighs nothing
  if (!known && warp == 0) {
    uint64_t rest_sum = lane < kHeadWarps ? s.red_low[lane] : 0, off = 0;
    if (lane < ctas) {
      // How far the bound lies below the largest, and the reference that the others were summed under, in octaves.  The reference is
      // the bound's product with c, rounded: `above` it by part of an octave or more where logits are large against T, or below.
      const double at = s.bound[lane], up = static_cast<double>(max_x) - at, above = s.ref[lane] - at * c_hi;
      const double fall = up * c_hi + up * c_lo, down = fall - above;
      if (fall < 60.0 && above > 0.125) {
        // The others were summed too coarsely: all that is taken of them is that each weighs no more than the bound.
        off = s.others[lane] * (weigh(s.bound[lane]) + 1);
      } else if (fall < 60.0 && down < 60.0) {  // (else they weigh nothing)
        const bool rises = down < 0.0;  // (by an eighth at most: an octave more, and back)
        const uint64_t tq = static_cast<uint64_t>((rises ? down + 1.0 : down) * 0x1p56);
        const uint64_t w =
            __umul64hi(s.rest[lane] << 17, exp2_fraction(tq, s.pow2)) >> ((rises ? 1 : 2) + static_cast<int>(tq >> 56));
        // Each weight is off by 2^-22 (ex2), seven additions, its argument's rounding and that of c, |t| (2^-24 + 2^-25) with
        // |t| 2^t at most 0.53 of the bound's weight and |t| up to an eighth larger for the reference, the sum's rounding to 2^-26
        // of 2^(1/8) of that weight (but for the first two, 2^-24 (ln 2 (0.53 1.5 + 1/8) + 2^(1/8) / 8) < 2^-24 of the bound's weight a
        // token), and half a unit when it is rounded to one.
        rest_sum += w;
        off = (w >> 20) + (s.others[lane] * weigh(s.bound[lane]) >> 24) + s.others[lane] / 2 + 2;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      rest_sum += __shfl_xor_sync(0xffffffffu, rest_sum, o);
      off += __shfl_xor_sync(0xffffffffu, off, o);
    }
    if (lane == 0) {
      s.rest_low = rest_sum > off ? rest_sum - off : 0;
      s.rest_high = rest_sum + off;
    }
  }
  __syncthreads();
  const uint64_t head = s.sum[n - 1];
  uint64_t low_all = head, high_all = head, total = head;
  if (!known) {
    low_all += s.rest_low;
    high_all += s.rest_high;
  }
  int32_t kept = n;
  bool decided = true;
  if (greedy || (k > 0 && k <= n)) {
    kept = greedy ? 1 : k;
    total = s.sum[kept - 1];
    known = true;
  } else if (k > 0 && !known) {
    decided = false;
  }
  const float p = a.top_p && !greedy ? a.top_p[r] : 1.0f;
  const float least = a.min_p && !greedy ? a.min_p[r] : 0.0f;
  if (decided && p < 1.0f) {
    uint64_t need[2];
    ask(s, need, known ? total : low_all, known ? total : high_all, [&](uint64_t whole) { return reaches(p, whole); });
    const int32_t m = first_place(s, n, need[0]);
    decided = need[1] <= head && s.sum[m] >= need[1];
    if (decided && m + 1 <= kept) {
      kept = m + 1;
      total = s.sum[m];
    }
    known = true;
  }
  if (decided && least > 0.0f) {
    if (tid == 0) s.low_w = least_of(least);
    __syncthreads();
    const int32_t m = first_light(s, n, s.low_w);
    if (m < kept) {
      kept = m;
      total = s.sum[m - 1];
      known = true;
    } else if (m == n && !known) {
      decided = false;
    }
  }
  if (decided) {
    uint64_t pass[2];
    const float u = a.u[r];
    ask(s, pass, known ? total : low_all, known ? total : high_all, [&](uint64_t whole) { return passes(u, whole); });
    const int32_t m = first_place(s, n, pass[0]);
    // (with a probability wanted, the weight that it is a part of has to be known to 2^-16)
    const bool near = known || !a.logprob || high_all - low_all <= low_all >> 15;
    if (near && pass[1] <= head && s.sum[m] >= pass[1]) {
      if (tid == 0) {
        a.tokens[r] = s.at[m];
        if (a.logprob)
          a.logprob[r] = ln_of(s.sum[m] - (m ? s.sum[m - 1] : 0), known ? total : low_all + (high_all - low_all) / 2);
      }
      return;
    }
  }
  if (tid == 0) a.tokens[r] = left_with(s.at[0]);
}

// A kernel whose launch may begin beside the end of the one ahead (it waits by itself), in clusters of `ctas`.
template <class S>
cudaError_t go(void (*kern)(SampleArgs), const SampleArgs& a, int64_t rows, int ctas, int threads, std::atomic<uint64_t>& ready,
               cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);  // ready: devices on which the kernel may use its shared memory
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(S)));
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(rows * ctas));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = sizeof(S);
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, a);
}

template <typename E>
cudaError_t run_sample(const SampleArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> ready[4];
  // CTAs a row.  Rows that one takes in a step of its pass have one (8,000 logits: 13.6 us, 14.2 by two).  Others as many as leave
  // the SMs a CTA each: 131,072 bf16 logits, 64 rows: 28.6 us by one, 25.2 by two, 26.6 by four; 100 rows: 29.4, 31.5, 35.6;
  // 16 rows: 25.6, 21.7, 19.0 and 19.6 by eight; 4 rows 16.9 by four, 15.6 by eight.
  int ctas = 1;
  if (a.V / Logit<E>::kVec >= 4 * kHeadThreads)
    while (ctas < kMostCtas && a.R * ctas * 2 <= (ctas == 4 ? 64 : 128)) ctas *= 2;
  const cudaError_t e = go<Head>(sample_head_kernel<E>, a, a.R, ctas, kHeadThreads, ready[0], st);
  if (e != cudaSuccess) return e;
  // Rows that are left: a cluster each, or, of many short rows, of which many may be, a CTA (300 flat rows of 3,000, 6,000, 12,000
  // and 24,000 bf16 logits: 46, 49, 63 and 86 us by CTAs, 138, 95, 115 and 124 by clusters; 300 of which none to two are left,
  // of 6,000, 12,000 and 24,000: 22, 30 and 52 against 24, 29 and 38; 30 flat rows of 12,000: 51 against 36).
  if (a.V <= 12288 && a.R >= 64)
    return go<Binned>(sample_binned_kernel<E, 1>, a, std::min<int64_t>(a.R, 152), 1, kThreads, ready[3], st);
  if (sizeof(E) == 2 && a.V <= kMostCounted)
    return go<Counts>(sample_counts_kernel, a, std::min<int64_t>(a.R, 152 / kCountPeers), kCountPeers, kCountThreads, ready[1], st);
  return go<Binned>(sample_binned_kernel<E, 8>, a, std::min<int64_t>(a.R, 152 / 8), 8, kThreads, ready[2], st);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, bool f32, cudaStream_t st) {
  return f32 ? run_sample<float>(a, st) : run_sample<uint16_t>(a, st);
}

}  // namespace catq
