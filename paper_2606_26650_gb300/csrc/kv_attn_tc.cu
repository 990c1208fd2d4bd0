// kv_attn_tc.cu — grouped-query attention of new tokens over the paged cache of 8-bit codes.
#include <cuda_fp16.h>

#include "launch.h"
#include "ptx_sm100.cuh"

namespace catq {
namespace {

constexpr int kThreads = 128;

// One warp per (row, query head), an online softmax over the row's cached tokens one by one.
__global__ void __launch_bounds__(kThreads) kv_attention_kernel(const KvAttnArgs a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = blockIdx.x;
  const int h = blockIdx.y * (kThreads / 32) + warp;
  int lo = 0, hi = a.B;  // the last sequence whose first row is not behind `row`
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.row_start[mid] <= row) lo = mid;
    else hi = mid;
  }
  const int b = lo;
  const int64_t r0 = a.row_start[b], r1 = a.row_start[b + 1];
  if (row < r0 || row >= r1 || h >= a.nh) return;
  const int32_t d = a.cache.d, page = a.cache.page, nkv = a.cache.nkv, hk = h / (a.nh / nkv), vpl = d / 32;
  const int64_t len = a.seq_len[b];
  if (r0 < 0 || r1 > a.T || len < 0 || len > static_cast<int64_t>(a.cache.max_pages) * page) {
    if (lane == 0) atomicCAS(a.status, 0, 10 /* CATQ_ERR_INDEX */);
    return;
  }
  const int64_t last = len - (r1 - r0) + (row - r0);
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.0f;
  for (int i = 0; i < vpl; ++i)
    q[i] = __uint_as_float(uint32_t(a.q[row * a.ldq + h * d + lane * vpl + i]) << 16) * a.scale_log2;
  for (int64_t j = 0; j <= last; ++j) {
    const int32_t id = a.cache.table[static_cast<int64_t>(b) * a.cache.max_pages + j / page];
    if (id < 0 || id >= a.cache.n_pages) {
      if (lane == 0) atomicCAS(a.status, 0, 10);
      continue;
    }
    const int64_t block = static_cast<int64_t>(id) * nkv + hk;
    const int64_t at = (block * page + j % page) * d + lane * vpl;
    auto value = [](uint8_t code) {
      uint32_t two;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(two) : "h"(static_cast<uint16_t>(code)));
      return __half2float(__ushort_as_half(static_cast<uint16_t>(two & 0xffffu)));
    };
    float s = 0.0f;
    for (int i = 0; i < vpl; ++i) s = fmaf(q[i], value(a.cache.k_codes[at + i]), s);
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= a.cache.k_scale[block];
    const float m_new = fmaxf(m, s);
    const float f = m == -INFINITY ? 0.0f : exp2f(m - m_new), p = s == -INFINITY ? 0.0f : exp2f(s - m_new);
    l = l * f + p;
    const float pv = p * a.cache.v_scale[block];
    for (int i = 0; i < vpl; ++i) o[i] = o[i] * f + pv * value(a.cache.v_codes[at + i]);
    m = m_new;
  }
  for (int i = 0; i < vpl; ++i) {
    const float v = l == 0.0f ? 0.0f : o[i] / l;
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(0.0f), "f"(v));
    a.o[row * a.ldo + h * d + lane * vpl + i] = static_cast<uint16_t>(r & 0xffffu);
  }
  if (a.lse && lane == 0) a.lse[row * a.nh + h] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

size_t kv_attention_ws_bytes(int32_t, int32_t, int32_t) { return 256; }

cudaError_t launch_kv_attention(KvAttnArgs a, cudaStream_t st) {
  WaitCtl wc;
  if (!launch_wait_ctl(&wc)) return cudaErrorInvalidDevice;
  a.status = wc.status_word;
  kv_attention_kernel<<<dim3(static_cast<unsigned>(a.T), (a.nh + 3) / 4), kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace catq
