// Position rotation of q and k, and the append of k and v to a paged cache as 8- or 4-bit
// codes with one scale per position and head.
//
// A value's 16-bit row (k rotated and rounded to the rows' type first, which is what a 16-bit
// cache would hold) has a = max |x|, s = fl32(a / m), m = 127 or 7, and codes
// round_half_even(fl32(x / s)). The rotation rounds each product and the sum to fp32, so that
// codes and scales follow from the rows bit for bit.
//
// As in the 16-bit append a thread takes 16 dimensions of a head, in two pieces, and the same
// place of several heads of one token; the 8 (dh 64: 4) threads of a head find its maximum by
// shuffles. The bound is HBM, and at a few tokens the chain of index, page, angle and store.
// 22528 tokens x 120 heads of 128 at 4 bits with the rows kept: 260 us, 0.86 of what a copy
// of as many bytes takes; one token 4.1 us, 96 tokens 3.3 us.
#include <cuda_runtime.h>

#include "p4q_codes.cuh"
#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {
namespace {

__device__ unsigned int g_rope_quant_err;

constexpr int kThreads = 256;
// Items per thread, at most: eight share the index, the page and the angles (22528 x 120 heads 260 us;
// four 288, sixteen 266 at four CTAs per SM).
constexpr int kItems = 8;
// CTAs per SM (four 269 us, six 264; the next head's loads ahead of this one's work: 273, at four 261)
constexpr int kResident = 5;

// Pairs (x, y) of four dimensions each turned by angles c, s, each operation rounded.
__device__ __forceinline__ float2 turned(float x, float y, float c, float s) {
  return make_float2(__fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s)), __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s)));
}

template <bool kBf16, bool kInter, int kBits>
__global__ void __launch_bounds__(kThreads, kResident) rope_append_quant_kernel(const RopeQuantArgs a, const int tx_log2) {
  const PagedCodes& c = a.kv;
  const int tx = 1 << tx_log2;  // threads per token
  const long long t = static_cast<long long>(blockIdx.x) * (kThreads >> tx_log2) + (threadIdx.x >> tx_log2);
  const int lane = threadIdx.x & (tx - 1);
  pdl_wait();
  pdl_launch_dependents();
  if (t >= a.T) return;
  const int per_log2 = c.dh == 128 ? 3 : 2;  // threads per head
  const int j = lane & ((1 << per_log2) - 1);
  const uint32_t mine = ((1u << (1 << per_log2)) - 1u) << (threadIdx.x & 31 & ~((1 << per_log2) - 1));  // the head's lanes
  const int step = tx >> per_log2;  // heads between a thread's items
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
    if (lane == 0) atomicOr(&g_rope_quant_err, kErrIndex);
    return;
  }
  const int in_page = p & ((1 << c.page_log2) - 1);
  const long long slot = page * c.page_stride + in_page * c.token_stride;
  const long long scale_slot = page * c.scale_page_stride + in_page * c.scale_token_stride;
  const long long angle = static_cast<long long>(rp) * (a.rot / 2) + 8 * j;

  // Heads of q, then of k, then of v, with a loop for each: what is the same for all of them stays out
  // of the loops (one loop that chose by the head: 333 instructions per item of a warp and 277 us).
  auto load = [&](const uint16_t* src, uint4& x, uint4& y) {
    x = ldg_stream16(src + lo);
    y = ldg_stream16(src + hi);
  };
  auto turn = [&](uint4& x, uint4& y) {
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
          const float2 u = unpack2<kBf16>(r[e]), w = turned(u.x, u.y, cs[e], sn[e]);
          r[e] = pack2<kBf16>(w.x, w.y);
        }
      } else {  // pairs across the pieces
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 u = unpack2<kBf16>(xr[2 * half + e]), w = unpack2<kBf16>(yr[2 * half + e]);
          const float2 d0 = turned(u.x, w.x, cs[2 * e], sn[2 * e]), d1 = turned(u.y, w.y, cs[2 * e + 1], sn[2 * e + 1]);
          xr[2 * half + e] = pack2<kBf16>(d0.x, d1.x);
          yr[2 * half + e] = pack2<kBf16>(d0.y, d1.y);
        }
      }
    }
    x = make_uint4(xr[0], xr[1], xr[2], xr[3]);
    y = make_uint4(yr[0], yr[1], yr[2], yr[3]);
  };
  // A row's codes to d, its scale to *scale_to, the values to back (which may be null)
  auto write = [&](const uint4& x, const uint4& y, uint8_t* d, float* scale_to, uint16_t* back) {
    const uint32_t w[2][4] = {{x.x, x.y, x.z, x.w}, {y.x, y.y, y.z, y.w}};
    uint32_t most = 0;  // |x| as bits: their order is that of the values, inf and NaN above all
#pragma unroll
    for (int e = 0; e < 4; ++e) most = __vmaxu2(most, __vmaxu2(w[0][e] & 0x7FFF7FFFu, w[1][e] & 0x7FFF7FFFu));
#pragma unroll
    for (int d = 1; d < 8; d <<= 1)
      if (d < (1 << per_log2)) most = __vmaxu2(most, __shfl_xor_sync(mine, most, d));
    most = max(most & 0xFFFFu, most >> 16);
    const bool finite = most < (kBf16 ? 0x7F80u : 0x7C00u);
    const QRowF q = quant_row_f(finite ? from16<kBf16>(static_cast<uint16_t>(most)) : 0.0f, kBits == 8 ? 127.0f : 7.0f);
    const bool divide = q.s > 0.0f && q.s < 0x1p-100f;
    const float scale = finite ? q.s : __int_as_float(0x7FFFFFFF);
    const uint32_t keep = finite ? 0xFFFFFFFFu : 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = i == 0 ? lo : hi;
      float2 f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = unpack2<kBf16>(w[i][e] & keep);
      uint32_t tb[8];
      quant_values(f, q, tb, divide);
      if (kBits == 8) {
        uint2 b;  // the low bytes in order
        b.x = __byte_perm(__byte_perm(tb[0], tb[1], 0x0040), __byte_perm(tb[2], tb[3], 0x0040), 0x5410);
        b.y = __byte_perm(__byte_perm(tb[4], tb[5], 0x0040), __byte_perm(tb[6], tb[7], 0x0040), 0x5410);
        __stcs(reinterpret_cast<uint2*>(d + at), b);
      } else {
        __stcs(reinterpret_cast<uint32_t*>(d + at / 2), packed4(gather_codes(tb)));
      }
      if (back) {
        uint32_t r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)  // (the magic number's codes as fp32: exact)
          r[e] = pack2<kBf16>((__uint_as_float(tb[2 * e]) - 12582912.0f) * scale,
                              (__uint_as_float(tb[2 * e + 1]) - 12582912.0f) * scale);
        __stcs(reinterpret_cast<uint4*>(back + at), make_uint4(r[0], r[1], r[2], r[3]));
      }
    }
    if (j == 0) *scale_to = scale;
  };
  int h = lane >> per_log2;
  const int across = step * c.dh;  // to the thread's next head, in a row
  {
    const uint16_t* src = a.q + t * a.ldq + h * c.dh;
    uint16_t* d = a.q_out + t * a.ldqo + h * c.dh;
#pragma unroll 1
    for (; h < a.H; h += step, src += across, d += across) {
      uint4 x, y;
      load(src, x, y);
      if (turns) turn(x, y);
      __stcs(reinterpret_cast<uint4*>(d + lo), x);
      __stcs(reinterpret_cast<uint4*>(d + hi), y);
    }
  }
  const long long code_step = step * c.head_stride, scale_step = step * c.scale_head_stride;
#pragma unroll
  for (int is_v = 0; is_v < 2; ++is_v) {
    const int hk = h - a.H - is_v * c.Hkv, end = a.H + (1 + is_v) * c.Hkv;
    const uint16_t* src = is_v ? a.v + t * a.ldv : a.k + t * a.ldk;
    uint16_t* back = is_v ? a.v_out : a.k_out;
    const bool rows = back != nullptr;
    if (rows) back += t * (is_v ? a.ldvo : a.ldko) + hk * c.dh;
    src += hk * c.dh;
    uint8_t* d = (is_v ? c.v : c.k) + slot + hk * c.head_stride;
    float* scale_to = (is_v ? c.v_scale : c.k_scale) + scale_slot + hk * c.scale_head_stride;
#pragma unroll 1
    for (; h < end; h += step, src += across, back += across, d += code_step, scale_to += scale_step) {
      uint4 x, y;
      load(src, x, y);
      if (!is_v && turns) turn(x, y);
      write(x, y, d, scale_to, rows ? back : nullptr);
    }
  }
}

template <int kBits>
cudaError_t launch_for(const RopeQuantArgs& a, cudaStream_t stream) {
  auto* kernel = a.bf16 ? (a.interleaved ? rope_append_quant_kernel<true, true, kBits> : rope_append_quant_kernel<true, false, kBits>)
                        : (a.interleaved ? rope_append_quant_kernel<false, true, kBits> : rope_append_quant_kernel<false, false, kBits>);
  // threads per token as in the 16-bit append
  const int items = (a.H + 2 * a.kv.Hkv) * (a.kv.dh / 16);
  int tx_log2 = 3;
  while (tx_log2 < 8 && ((kItems << tx_log2) < items || ((1 << tx_log2) < items && a.T <= (num_sms() * kThreads) >> tx_log2)))
    ++tx_log2;
  const unsigned tokens = kThreads >> tx_log2;
  return launch_pdl(kernel, dim3((static_cast<unsigned>(a.T) + tokens - 1) / tokens), dim3(kThreads), 0, stream, a, tx_log2);
}

}  // namespace

cudaError_t launch_rope_append_quant(const RopeQuantArgs& a, cudaStream_t stream) {
  return a.kv.bits == 8 ? launch_for<8>(a, stream) : launch_for<4>(a, stream);
}

unsigned int rope_quant_read_and_clear_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_rope_quant_err, sizeof(v));
  cudaMemcpyToSymbol(g_rope_quant_err, &z, sizeof(z));
  return v;
}

}  // namespace p4q
