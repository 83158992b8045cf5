// The draw of one token from each row of logits: temperature, top-k, top-p and
// min-p with a given uniform number.
//
// Weights are integers (2^31 exp(-d) rounded), so that their sums are exact and
// the drawn token depends on no order of summation. The kept tokens are a head
// of the row sorted by falling logit and rising index, so each cut is a last
// token (its key and index); a radix walk over the logits' ordered bit patterns
// finds it from counts (top-k) or weights (top-p).
#include <climits>
#include <cuda_runtime.h>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {
namespace {

constexpr int kThreads = 1024;
typedef unsigned long long u64;

template <int kType>
__device__ __forceinline__ float logit(const void* row, int i) {
  float x;
  if (kType == 2) x = static_cast<const float*>(row)[i];
  else x = from16<kType == 1>(static_cast<const uint16_t*>(row)[i]);
  return x != x ? -INFINITY : x + 0.0f;  // NaN as -inf, -0 as +0
}

// Larger floats have larger keys.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

struct Cut {  // the last kept token: keys above, and this key up to the index
  uint32_t key;
  int idx;
  __device__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= idx); }
};

struct Shared {
  u64 hist[256];
  u64 scan[kThreads / 32 + 1];
  u64 rest;
  uint32_t prefix;
  uint32_t umax;
  int imin;
};

// Inclusive scan over the block's threads; *total the sum.
__device__ u64 block_scan(u64 v, Shared& s, u64* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 u = __shfl_up_sync(0xFFFFFFFFu, v, d);
    if (lane >= d) v += u;
  }
  __syncthreads();
  if (lane == 31) s.scan[warp] = v;
  __syncthreads();
  u64 before = 0, all = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += s.scan[w];
    all += s.scan[w];
  }
  *total = all;
  return v + before;
}

template <int kType>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ Shared s;
  const int n = blockIdx.x, V = a.vocab, t = threadIdx.x;
  const void* row = static_cast<const char*>(a.logits) + n * a.ld * (kType == 2 ? 4 : 2);
  // the row's largest logit and its first index
  if (t == 0) {
    s.umax = 0;
    s.imin = INT_MAX;
  }
  __syncthreads();
  uint32_t mine = 0;
  for (int i = t; i < V; i += kThreads) mine = max(mine, key_of(logit<kType>(row, i)));
  atomicMax(&s.umax, mine);
  __syncthreads();
  const uint32_t kmax = s.umax;
  const float xmax = __uint_as_float((kmax & 0x80000000u) ? kmax & 0x7FFFFFFFu : ~kmax);
  if (xmax == -INFINITY) {
    if (t == 0) {
      a.token[n] = -1;
      if (a.logprob) a.logprob[n] = -INFINITY;
    }
    return;
  }
  const float temp = a.temperature ? a.temperature[n] : 1.0f;
  if (!(temp > 0.0f)) {
    for (int i = t; i < V; i += kThreads)
      if (key_of(logit<kType>(row, i)) == kmax) atomicMin(&s.imin, i);
    __syncthreads();
    if (t == 0) {
      a.token[n] = s.imin;
      if (a.logprob) a.logprob[n] = 0.0f;
    }
    return;
  }
  const float inv_t = 1.0f / temp;
  auto dist = [&](float x) { return x == xmax ? 0.0f : (xmax - x) * inv_t; };
  auto weight = [&](float x) { return static_cast<u64>(__float2ull_rn(expf(-dist(x)) * 2147483648.0f)); };
  const int chunk = (V + kThreads - 1) / kThreads, i0 = min(V, t * chunk), i1 = min(V, i0 + chunk);
  Cut cut{0u, INT_MAX};
  // Shortens the kept head to the first tokens whose counts (by_mass false) or
  // weights reach `need` >= 1 (they do).
  auto shorten = [&](bool by_mass, u64 need) {
    uint32_t prefix = 0, mask = 0;
    for (int level = 24; level >= 0; level -= 8) {
      if (t < 256) s.hist[t] = 0;
      __syncthreads();
      for (int i = t; i < V; i += kThreads) {
        const float x = logit<kType>(row, i);
        const uint32_t k = key_of(x);
        if ((k & mask) == prefix && cut.keeps(k, i)) atomicAdd(&s.hist[(k >> level) & 255u], by_mass ? weight(x) : 1ull);
      }
      __syncthreads();
      if (t == 0) {
        int bin = 255;
        while (bin > 0 && s.hist[bin] < need) need -= s.hist[bin--];
        s.prefix = prefix | (static_cast<uint32_t>(bin) << level);
        s.rest = need;
      }
      __syncthreads();
      prefix = s.prefix;
      need = s.rest;
      mask |= 0xFFu << level;
      __syncthreads();
    }
    // among equal logits, by index
    u64 c = 0;
    const float x = __uint_as_float((prefix & 0x80000000u) ? prefix & 0x7FFFFFFFu : ~prefix);
    const u64 each = by_mass ? weight(x) : 1ull;
    for (int i = i0; i < i1; ++i) {
      const uint32_t k = key_of(logit<kType>(row, i));
      if (k == prefix && cut.keeps(k, i)) c += each;
    }
    u64 total;
    const u64 upto = block_scan(c, s, &total);
    if (t == 0) s.imin = INT_MAX;
    __syncthreads();
    if (c > 0 && upto >= need && upto - c < need) {
      u64 at = upto - c;
      for (int i = i0; i < i1; ++i) {
        const uint32_t k = key_of(logit<kType>(row, i));
        if (k == prefix && cut.keeps(k, i) && (at += each) >= need) {
          s.imin = i;
          break;
        }
      }
    }
    __syncthreads();
    cut.key = prefix;
    cut.idx = s.imin;
    __syncthreads();
  };
  const int top_k = a.top_k ? a.top_k[n] : 0;
  if (top_k > 0 && top_k < V) shorten(false, static_cast<u64>(top_k));
  const float top_p = a.top_p ? a.top_p[n] : 1.0f;
  u64 total;
  if (top_p < 1.0f) {
    u64 c = 0;
    for (int i = t; i < V; i += kThreads) {
      const float x = logit<kType>(row, i);
      if (cut.keeps(key_of(x), i)) c += weight(x);
    }
    block_scan(c, s, &total);
    __syncthreads();
    const double need = ceil(static_cast<double>(top_p) * static_cast<double>(total));
    shorten(true, need < 1.0 ? 1ull : static_cast<u64>(need));
  }
  const float min_p = a.min_p && a.min_p[n] > 0.0f ? fminf(a.min_p[n], 1.0f) : 0.0f;
  auto kept = [&](float x, int i) { return cut.keeps(key_of(x), i) && !(expf(-dist(x)) < min_p); };
  u64 c = 0;
  for (int i = i0; i < i1; ++i) {
    const float x = logit<kType>(row, i);
    if (kept(x, i)) c += weight(x);
  }
  const u64 upto = block_scan(c, s, &total);
  const double want = floor(static_cast<double>(a.u[n]) * static_cast<double>(total));
  u64 r = want > 0.0 ? static_cast<u64>(want) : 0ull;
  if (r > total - 1) r = total - 1;
  if (upto > r && upto - c <= r) {
    u64 at = upto - c;
    for (int i = i0; i < i1; ++i) {
      const float x = logit<kType>(row, i);
      if (kept(x, i) && (at += weight(x)) > r) {
        a.token[n] = i;
        if (a.logprob) a.logprob[n] = -dist(x) - logf(static_cast<float>(static_cast<double>(total) * 4.656612873077393e-10));
        break;
      }
    }
  }
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, cudaStream_t stream) {
  auto* kernel = a.dtype == 2 ? sample_kernel<2> : a.dtype == 1 ? sample_kernel<1> : sample_kernel<0>;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(a.rows)), dim3(kThreads), 0, stream, a);
}

}  // namespace p4q
