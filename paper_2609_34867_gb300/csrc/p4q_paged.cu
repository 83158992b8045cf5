// Attention of one new token per sequence over a paged key/value cache.
#include <cuda_runtime.h>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {

__device__ unsigned int g_paged_err;

namespace {

constexpr int kWarps = 8;

// One CTA per (sequence, head); each warp takes every eighth key with a running
// maximum and sum, a lane dh / 32 dimensions; the warps are joined at the end.
template <bool kBf16, int kDh>
__global__ void __launch_bounds__(kWarps * 32) paged_attention_kernel(const PagedAttnArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const PagedCache& c = a.kv;
  const int h = blockIdx.x, b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int hk = h / (a.H / c.Hkv);
  constexpr int kE = kDh / 32;
  int len = a.lens[b];
  const long long room = static_cast<long long>(c.table_cols) << c.page_log2;
  if (len > room) {
    len = static_cast<int>(room);
    if (threadIdx.x == 0) atomicOr(&g_paged_err, kErrIndex);
  }
  float q[kE], o[kE], m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    q[e] = from16<kBf16>(a.q[b * a.ldq + h * kDh + lane * kE + e]);
    o[e] = 0.0f;
  }
  for (int j = warp; j < len; j += kWarps) {
    const int page = c.table[static_cast<long long>(b) * c.table_ld + (j >> c.page_log2)];
    if (page < 0 || page >= c.pages) {
      if (lane == 0) atomicOr(&g_paged_err, kErrIndex);
      continue;
    }
    const long long at = page * c.page_stride + (j & ((1 << c.page_log2) - 1)) * c.token_stride + hk * c.head_stride + lane * kE;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) s = fmaf(q[e], from16<kBf16>(c.k[at + e]), s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    s *= a.scale;
    const float mx = fmaxf(m, s);
    const float al = m == -INFINITY ? 0.0f : expf(m - mx);
    const float p = expf(s - mx);
    m = mx;
    l = l * al + p;
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = o[e] * al + p * from16<kBf16>(c.v[at + e]);
  }
  __shared__ float sm[kWarps], sl[kWarps], so[kWarps][kDh];
  if (lane == 0) {
    sm[warp] = m;
    sl[warp] = l;
  }
#pragma unroll
  for (int e = 0; e < kE; ++e) so[warp][lane * kE + e] = o[e];
  __syncthreads();
  if (warp == 0) {
    float mx = -INFINITY, sum = 0.0f, acc[kE] = {};
    for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, sm[w]);
    for (int w = 0; w < kWarps; ++w) {
      const float f = sl[w] == 0.0f ? 0.0f : expf(sm[w] - mx);
      sum += f * sl[w];
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[e] += f == 0.0f ? 0.0f : f * so[w][lane * kE + e];
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < kE; e += 2)
      *reinterpret_cast<uint32_t*>(a.o + b * a.ldo + h * kDh + lane * kE + e) =
          pack2<kBf16>(acc[e] * inv, acc[e + 1] * inv);
    if (lane == 0 && a.lse) a.lse[static_cast<long long>(b) * a.H + h] = sum == 0.0f ? -INFINITY : mx + logf(sum);
  }
}

}  // namespace

size_t paged_attention_workspace_bytes() { return 16; }

cudaError_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t stream) {
  auto* kernel = a.kv.bf16 ? (a.kv.dh == 64 ? paged_attention_kernel<true, 64> : paged_attention_kernel<true, 128>)
                           : (a.kv.dh == 64 ? paged_attention_kernel<false, 64> : paged_attention_kernel<false, 128>);
  return launch_pdl(kernel, dim3(static_cast<unsigned>(a.H), static_cast<unsigned>(a.kv.seqs)), dim3(kWarps * 32), 0,
                    stream, a);
}

unsigned int paged_read_and_clear_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_paged_err, sizeof(v));
  cudaMemcpyToSymbol(g_paged_err, &z, sizeof(z));
  return v;
}

}  // namespace p4q
