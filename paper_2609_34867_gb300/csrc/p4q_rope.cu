// Position rotation of q and k, and the append of k and v to a paged cache.
//
// Per token and head, pair j of dimensions (a, b) turns by the angle whose
// cosine and sine the caller's tables hold: (x_a c - x_b s, x_b c + x_a s).
// Every row is read and written once: the bound is HBM, and at a few tokens the
// chain of index, page, angle and store.
//
// An item is 16 dimensions of a head (8 pairs), two 16-byte pieces. A thread
// takes the same place j of several heads of one token, one after the other, and
// a CTA as many tokens as its threads cover with about four items each. Many
// threads with little in flight each are faster than few with much: 22528 tokens
// of 40 heads with the rotated key rows kept too (1.63 GB) take 244 us (0.98 of the
// measured copy) at 40 registers (8 - 12 bytes of them spilled), 308 with four items
// loaded at once and the angles in registers (98). Stores are marked evict-first (249
// without, in the same call); of so many rows of q_out and k_out most have left L2 either
// way before the next kernel reads them.
#include <cuda_runtime.h>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {

__device__ unsigned int g_rope_err;

namespace {

constexpr int kThreads = 256;
constexpr int kItems = 4;  // per thread, at most

template <bool kBf16, bool kInter>
__global__ void __launch_bounds__(kThreads, 6) rope_append_kernel(const RopeArgs a, const int tx_log2) {
  const PagedCache& c = a.kv;
  const int tx = 1 << tx_log2;  // threads per token
  const long long t = static_cast<long long>(blockIdx.x) * (kThreads >> tx_log2) + (threadIdx.x >> tx_log2);
  const int lane = threadIdx.x & (tx - 1);
  pdl_wait();
  pdl_launch_dependents();
  if (t >= a.T) return;
  const int per_log2 = c.dh == 128 ? 3 : 2;  // items per head
  const int j = lane & ((1 << per_log2) - 1);
  const int heads = a.H + 2 * c.Hkv, step = tx >> per_log2;  // heads between a thread's items
  const bool turns = j < a.rot / 16;
  const int lo = turns && !kInter ? 8 * j : 16 * j;  // the pieces' dimensions (of v: any two of the item)
  const int hi = turns && !kInter ? 8 * j + a.rot / 2 : 16 * j + 8;

  const int p = a.pos[t];
  if (p < 0) return;
  const int sq = a.seq ? a.seq[t] : static_cast<int>(t);
  const int rp = a.rot_pos ? a.rot_pos[t] : p;
  const int col = p >> c.page_log2;
  int page = -1;
  if (sq >= 0 && sq < c.seqs && col < c.table_cols && rp >= 0 && rp < a.max_pos)
    page = c.table[static_cast<long long>(sq) * c.table_ld + col];
  if (page < 0 || page >= c.pages) {
    if (lane == 0) atomicOr(&g_rope_err, kErrIndex);
    return;
  }
  const long long slot = page * c.page_stride + (p & ((1 << c.page_log2) - 1)) * c.token_stride;
  const long long angle = static_cast<long long>(rp) * (a.rot / 2) + 8 * j;

#pragma unroll 1
  for (int h = lane >> per_log2; h < heads; h += step) {
    const bool is_q = h < a.H, is_v = h >= a.H + c.Hkv;
    const int hk = h - (is_q ? 0 : is_v ? a.H + c.Hkv : a.H);
    const uint16_t* src = (is_q ? a.q : is_v ? a.v : a.k) + t * (is_q ? a.ldq : is_v ? a.ldv : a.ldk) + hk * c.dh;
    uint4 x = ldg_stream16(src + lo), y = ldg_stream16(src + hi);
    if (turns && !is_v) {
      uint32_t xr[4] = {x.x, x.y, x.z, x.w}, yr[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // four pairs each
        const float4 c4 = *reinterpret_cast<const float4*>(a.cos + angle + 4 * half);
        const float4 s4 = *reinterpret_cast<const float4*>(a.sin + angle + 4 * half);
        const float cs[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
        if (kInter) {  // pairs within a piece
          uint32_t* r = half == 0 ? xr : yr;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 u = unpack2<kBf16>(r[e]);
            r[e] = pack2<kBf16>(u.x * cs[e] - u.y * sn[e], u.y * cs[e] + u.x * sn[e]);
          }
        } else {  // pairs across the pieces
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 u = unpack2<kBf16>(xr[2 * half + e]), w = unpack2<kBf16>(yr[2 * half + e]);
            xr[2 * half + e] = pack2<kBf16>(u.x * cs[2 * e] - w.x * sn[2 * e], u.y * cs[2 * e + 1] - w.y * sn[2 * e + 1]);
            yr[2 * half + e] = pack2<kBf16>(w.x * cs[2 * e] + u.x * sn[2 * e], w.y * cs[2 * e + 1] + u.y * sn[2 * e + 1]);
          }
        }
      }
      x = make_uint4(xr[0], xr[1], xr[2], xr[3]);
      y = make_uint4(yr[0], yr[1], yr[2], yr[3]);
    }
    uint16_t* d = is_q ? a.q_out + t * a.ldqo + hk * c.dh : (is_v ? c.v : c.k) + slot + hk * c.head_stride;
    __stcs(reinterpret_cast<uint4*>(d + lo), x);
    __stcs(reinterpret_cast<uint4*>(d + hi), y);
    if (!is_q && !is_v && a.k_out) {
      d = a.k_out + t * a.ldko + hk * c.dh;
      __stcs(reinterpret_cast<uint4*>(d + lo), x);
      __stcs(reinterpret_cast<uint4*>(d + hi), y);
    }
  }
}

}  // namespace

cudaError_t launch_rope_append(const RopeArgs& a, cudaStream_t stream) {
  auto* kernel = a.kv.bf16 ? (a.interleaved ? rope_append_kernel<true, true> : rope_append_kernel<true, false>)
                           : (a.interleaved ? rope_append_kernel<false, true> : rope_append_kernel<false, false>);
  // threads per token: a power of two of at least a quarter of its items, more
  // (up to one per item) while there are fewer CTAs than SMs (96 tokens x 48 heads
  // 3.0 -> 2.5 us, 22528 tokens x 48 with two items a thread 107 instead of 93)
  const int items = (a.H + 2 * a.kv.Hkv) * (a.kv.dh / 16);
  int tx_log2 = 3;
  while (tx_log2 < 8 && ((kItems << tx_log2) < items || ((1 << tx_log2) < items && a.T <= (num_sms() * kThreads) >> tx_log2)))
    ++tx_log2;
  const unsigned tokens = kThreads >> tx_log2;
  return launch_pdl(kernel, dim3((static_cast<unsigned>(a.T) + tokens - 1) / tokens), dim3(kThreads), 0, stream, a,
                    tx_log2);
}

unsigned int rope_read_and_clear_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_rope_err, sizeof(v));
  cudaMemcpyToSymbol(g_rope_err, &z, sizeof(z));
  return v;
}

}  // namespace p4q
