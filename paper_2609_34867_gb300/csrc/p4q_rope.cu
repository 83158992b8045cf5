// Position rotation of q and k, and the append of k and v to a paged cache.
//
// Per token and head, pair j of dimensions (a, b) turns by the angle whose
// cosine and sine the caller's tables hold: (x_a c - x_b s, x_b c + x_a s).
// Every row is read and written once.
#include <cuda_runtime.h>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {

__device__ unsigned int g_rope_err;

namespace {

constexpr int kThreads = 256;

// One CTA per token; an item is 16 dimensions of a head (8 pairs), two 16-byte
// pieces: dimensions lo .. lo + 7 and hi .. hi + 7.
template <bool kBf16, bool kInter>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const RopeArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const long long t = blockIdx.x;
  const PagedCache& c = a.kv;
  const int p = a.pos[t];
  if (p < 0) return;
  const int sq = a.seq ? a.seq[t] : static_cast<int>(t);
  const int rp = a.rot_pos ? a.rot_pos[t] : p;
  const int col = p >> c.page_log2;
  bool ok = sq >= 0 && sq < c.seqs && col < c.table_cols && rp >= 0 && rp < a.max_pos;
  int page = -1;
  if (ok) page = c.table[static_cast<long long>(sq) * c.table_ld + col];
  ok = page >= 0 && page < c.pages;
  if (!ok) {
    if (threadIdx.x == 0) atomicOr(&g_rope_err, kErrIndex);
    return;
  }
  const long long slot = page * c.page_stride + (p & ((1 << c.page_log2) - 1)) * c.token_stride;
  const int per = c.dh / 16;  // items per head
  const int items = (a.H + 2 * c.Hkv) * per;
  for (int i = threadIdx.x; i < items; i += kThreads) {
    const int h = i / per, j = i % per;
    const bool is_q = h < a.H, is_v = h >= a.H + c.Hkv;
    const int hk = is_v ? h - a.H - c.Hkv : h - a.H;
    const bool turn = !is_v && j < a.rot / 16;
    int lo = 16 * j, hi = 16 * j + 8;
    if (turn && !kInter) {
      lo = 8 * j;
      hi = 8 * j + a.rot / 2;
    }
    const uint16_t* src = is_q ? a.q + t * a.ldq + h * c.dh : is_v ? a.v + t * a.ldv + hk * c.dh : a.k + t * a.ldk + hk * c.dh;
    uint4 x = *reinterpret_cast<const uint4*>(src + lo), y = *reinterpret_cast<const uint4*>(src + hi);
    if (turn) {
      uint32_t xr[4] = {x.x, x.y, x.z, x.w}, yr[4] = {y.x, y.y, y.z, y.w};
      const float* cs = a.cos + static_cast<long long>(rp) * (a.rot / 2) + 8 * j;
      const float* sn = a.sin + static_cast<long long>(rp) * (a.rot / 2) + 8 * j;
      if (kInter) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 u = unpack2<kBf16>(xr[e]), w = unpack2<kBf16>(yr[e]);
          xr[e] = pack2<kBf16>(u.x * cs[e] - u.y * sn[e], u.y * cs[e] + u.x * sn[e]);
          yr[e] = pack2<kBf16>(w.x * cs[4 + e] - w.y * sn[4 + e], w.y * cs[4 + e] + w.x * sn[4 + e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 u = unpack2<kBf16>(xr[e]), w = unpack2<kBf16>(yr[e]);
          const float c0 = cs[2 * e], c1 = cs[2 * e + 1], s0 = sn[2 * e], s1 = sn[2 * e + 1];
          xr[e] = pack2<kBf16>(u.x * c0 - w.x * s0, u.y * c1 - w.y * s1);
          yr[e] = pack2<kBf16>(w.x * c0 + u.x * s0, w.y * c1 + u.y * s1);
        }
      }
      x = make_uint4(xr[0], xr[1], xr[2], xr[3]);
      y = make_uint4(yr[0], yr[1], yr[2], yr[3]);
    }
    if (is_q) {
      uint16_t* d = a.q_out + t * a.ldqo + h * c.dh;
      *reinterpret_cast<uint4*>(d + lo) = x;
      *reinterpret_cast<uint4*>(d + hi) = y;
    } else {
      uint16_t* d = (is_v ? c.v : c.k) + slot + hk * c.head_stride;
      *reinterpret_cast<uint4*>(d + lo) = x;
      *reinterpret_cast<uint4*>(d + hi) = y;
      if (!is_v && a.k_out) {
        d = a.k_out + t * a.ldko + hk * c.dh;
        *reinterpret_cast<uint4*>(d + lo) = x;
        *reinterpret_cast<uint4*>(d + hi) = y;
      }
    }
  }
}

}  // namespace

cudaError_t launch_rope_append(const RopeArgs& a, cudaStream_t stream) {
  auto* kernel = a.kv.bf16 ? (a.interleaved ? rope_append_kernel<true, true> : rope_append_kernel<true, false>)
                           : (a.interleaved ? rope_append_kernel<false, true> : rope_append_kernel<false, false>);
  return launch_pdl(kernel, dim3(static_cast<unsigned>(a.T)), dim3(kThreads), 0, stream, a);
}

unsigned int rope_read_and_clear_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_rope_err, sizeof(v));
  cudaMemcpyToSymbol(g_rope_err, &z, sizeof(z));
  return v;
}

}  // namespace p4q
