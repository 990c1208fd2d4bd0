// tree.cu — trees of drafted tokens: what each token sees of the others (catq_tree_masks) and the branch that agrees with
// the tokens drawn (catq_tree_accept).
#include <cuda_runtime.h>

#include "launch.h"
#include "ptx_sm100.cuh"

namespace catq {
namespace {

__device__ __forceinline__ void latch_index_error(int32_t* status) { atomicCAS(status, 0, 10 /* CATQ_ERR_INDEX */); }

// A sequence's rows; none (latched) where the offsets are out of range.
struct Span {
  int32_t r0, n, len;
};
__device__ __forceinline__ Span span_of(const int32_t* row_start, const int32_t* seq_len, int32_t b, int64_t T, int32_t most,
                                        int32_t* status) {
  Span s;
  s.r0 = row_start[b];
  const int32_t r1 = row_start[b + 1];
  s.len = seq_len[b];
  s.n = r1 - s.r0;
  if (s.r0 < 0 || r1 < s.r0 || r1 > T || s.len < 0 || s.n > most) {
    if ((threadIdx.x & 31) == 0) latch_index_error(status);
    s.n = 0;
  }
  return s;
}

struct MaskArgs {
  const int32_t *parent, *row_start, *seq_len;
  int64_t T;
  uint32_t* seen;
  int32_t* positions;
  int32_t* status;
};

// A CTA a sequence, a thread a row: its bits and those of the row it has reached, twice as far up each time.  Bound by latency (a
// launch, two dependent loads, as many barriers as the depth has bits): one tree of 8 rows 1.6 us, 256 of up to 127 2.3.
template <int W>
__global__ void __launch_bounds__(32 * W) tree_masks_kernel(const MaskArgs a) {
  __shared__ uint32_t bits[32 * W][W];
  __shared__ int32_t up[32 * W];
  const Span s = span_of(a.row_start, a.seq_len, blockIdx.x, a.T, 32 * W, a.status);
  const int i = threadIdx.x;
  int32_t p = -1;
  if (i < s.n) {
    p = a.parent[s.r0 + i];
    if (p >= i) {  // a parent comes before its children
      latch_index_error(a.status);
      p = -1;
    }
    p = max(p, -1);
  }
  uint32_t m[W];
#pragma unroll
  for (int w = 0; w < W; ++w) m[w] = i >> 5 == w ? 1u << (i & 31) : 0u;
  while (__syncthreads_or(p >= 0)) {
#pragma unroll
    for (int w = 0; w < W; ++w) bits[i][w] = m[w];
    up[i] = p;
    __syncthreads();
    if (p >= 0) {
#pragma unroll
      for (int w = 0; w < W; ++w) m[w] |= bits[p][w];
      p = up[p];
    }
  }
  if (i >= s.n) return;
  int32_t depth = -1;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    a.seen[(static_cast<int64_t>(s.r0) + i) * W + w] = m[w];
    depth += __popc(m[w]);
  }
  if (a.positions) a.positions[s.r0 + i] = s.len - s.n + depth;
}

constexpr int kAcceptWarps = 4;

// A warp a sequence.  Children come behind their parents, so one sweep over the rows meets every row of the branch in
// order: the next is the first row of the rest whose parent is the last one and whose token was drawn there.  Bound by latency:
// 1.9 us for one tree of 8 rows, 2.9 for 256 of up to 127.
__global__ void __launch_bounds__(32 * kAcceptWarps) tree_accept_kernel(const TreeAcceptArgs a) {
  const int lane = threadIdx.x & 31;
  const int32_t b = blockIdx.x * kAcceptWarps + (threadIdx.x >> 5);
  if (b >= a.B) return;
  const Span s = span_of(a.row_start, a.seq_len, b, a.T, 0x7fffffff, a.status);
  int32_t last = 0, token = -1, count = 0;
  if (s.n > 0) {
    token = a.sampled[s.r0];
    count = 1;
    if (lane == 0) a.path[s.r0] = 0;
  }
#pragma unroll 1
  for (int32_t c = 0; c < s.n; c += 32) {
    const int32_t i = c + lane;
    int32_t parent = -1, drafted = -1, sampled = -1;
    if (i < s.n) {
      parent = a.parent[s.r0 + i];
      drafted = a.drafted[s.r0 + i];
      sampled = a.sampled[s.r0 + i];
    }
#pragma unroll 1
    for (;;) {
      const uint32_t fits = __ballot_sync(0xffffffffu, i > last && parent == last && drafted == token && drafted >= 0);
      if (!fits) break;
      const int l = __ffs(fits) - 1;
      last = c + l;
      token = __shfl_sync(0xffffffffu, sampled, l);
      if (lane == 0) a.path[s.r0 + count] = last;
      ++count;
    }
  }
  for (int32_t k = count + lane; k < s.n; k += 32) a.path[s.r0 + k] = -1;
  if (lane == 0) {
    a.n_kept[b] = count;
    a.next[b] = token;
    a.new_len[b] = s.len - s.n + count;
  }
}

}  // namespace

cudaError_t launch_tree_masks(const int32_t* parent, const int32_t* row_start, const int32_t* seq_len, int32_t B, int64_t T,
                              uint32_t* seen, int32_t words, int32_t* positions, cudaStream_t st) {
  WaitCtl wc;
  if (!launch_wait_ctl(&wc)) return cudaErrorInvalidDevice;
  const MaskArgs a{parent, row_start, seq_len, T, seen, positions, wc.status_word};
  switch (words) {
    case 1: tree_masks_kernel<1><<<B, 32, 0, st>>>(a); break;
    case 2: tree_masks_kernel<2><<<B, 64, 0, st>>>(a); break;
    case 3: tree_masks_kernel<3><<<B, 96, 0, st>>>(a); break;
    case 4: tree_masks_kernel<4><<<B, 128, 0, st>>>(a); break;
    case 5: tree_masks_kernel<5><<<B, 160, 0, st>>>(a); break;
    case 6: tree_masks_kernel<6><<<B, 192, 0, st>>>(a); break;
    case 7: tree_masks_kernel<7><<<B, 224, 0, st>>>(a); break;
    default: tree_masks_kernel<8><<<B, 256, 0, st>>>(a);
  }
  return cudaGetLastError();
}

cudaError_t launch_tree_accept(TreeAcceptArgs a, cudaStream_t st) {
  WaitCtl wc;
  if (!launch_wait_ctl(&wc)) return cudaErrorInvalidDevice;
  a.status = wc.status_word;
  tree_accept_kernel<<<(a.B + kAcceptWarps - 1) / kAcceptWarps, 32 * kAcceptWarps, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace catq
