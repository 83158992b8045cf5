// Attention of one new token per sequence over a paged key/value cache:
//   o_h = sum_{j < len} p_j v_j,  p = softmax_j(scale q_h . k_j).
//
// Work: a unit is one key/value head of one sequence with up to 8 NT of the
// query heads that share it (a group of more heads makes several units), cut
// into tiles of positions. Few units: each is a cluster's, and its CTAs'
// parts are added up in the first one's shared memory. Else all units' tiles in one
// row, unit after unit, are dealt to the CTAs in equal consecutive ranges, so a
// CTA's work does not depend on how unequal the sequences are (few tiles: one piece
// of a unit per CTA); the units that several CTAs share are joined by a second kernel.
//
// A warp takes 16 positions at a time, straight from global memory into the
// operands of m16n8k16 tensor-core products, without shared memory: the
// positions are the rows of S^T = K Q^T and the inner axis of O^T = V^T P^T.
//   K: lane (g, t) = (lane / 4, lane % 4) loads 16 bytes (8 dimensions) of rows
//      g and g + 8; which dimension an MMA calls its k-th is free as long as Q
//      has them in the same order, so these bytes are the operand as they lie.
//   V: the lane loads 16 bytes of positions 2t, 2t + 1, 2t + 8, 2t + 9; byte
//      permutations pair the positions of one dimension.
//   P: S^T leaves the first product with positions as rows; movmatrix turns it
//      into the second one's operand.
// The reference maximum of the softmax moves only when a score exceeds it by
// 2^8 (fp16 2^4: p stays below 2^15), so that most tiles need no exchange between lanes.
// p goes into the product as the sum of 16-bit values: two in fp16 (22 bits), three in
// bf16 (24 bits, all of p). Rounded once it would add as much error as the output's own
// rounding does. Two of bf16 leave 0.24 % of the outputs of 128 sequences of up to 8190 a
// rounding away from fp32 arithmetic's, three 0.10 %, for 0.4 % of the time (165.8 and 166.4
// us; 3 - 9 % where instructions are the bound: 12 and 16 heads per key/value head, pages of
// 1 and 8). None of the values of a p > 0 is negative or 0, so that an
// infinite value in V stays infinite.
// The new keys' loads are issued as soon as the old ones are in the first
// product, and the values' behind the second: 8 KB in flight per warp, twelve
// warps per SM. (Sixteen at 128 registers spilled: 757 us for 64 sequences of
// 16384 x 8 heads, 631 this way. Copies into shared memory two tiles ahead left
// room for eight warps, which their products' and exchanges' latencies bound: 907.)
//
// Bound: HBM. Times among other calls, on the GPU. 64 x 16384 positions, 32 heads over 8 of
// 128, bf16, pages of 16 (4.3 GB): 606 - 628 us = 6.8 - 7.1 TB/s, the measured copy (6.78); of
// 8 the same, of 1 727; of 64 dimensions 314 - 348 (pages of 8 381 - 390); 12 or 16 heads per key/value
// head, 4 of these, 353 (pages of 8 414: instructions). 24 sequences of up to 2048 x 40 heads 82 - 85 us
// = 0.92 of the copy, 128 of up to 8190 (skewed) x 8 167 - 171 = 0.96; one of 32011 x 8 28.4 = 0.68. Short ones
// cost a chain: lengths, page numbers, keys 4.6 us, then the end of a kernel and the second
// kernel 4, or the cluster's exchange 1.5: one of 704 x 40 6.2 us (by ranges 9.4), of 512 x 8
// 3.9 (6.9), 10 of 1024 x 8 11.0 (15.8).
#include <cuda_runtime.h>

#include <algorithm>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {

__device__ unsigned int g_paged_err;

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxGrid = 640;    // CTAs of a launch at most (partial results of the workspace)
constexpr int kMinTiles = 2;     // tiles per CTA at least, of one unit
constexpr int kUnitCost = 2;     // what a unit costs beside its tiles, in tiles
constexpr int kMaxCluster = 8;   // CTAs that share a unit as a cluster
constexpr int kJoinTiles = 8;    // what the second kernel costs, in tiles of a CTA
constexpr long long kMaxLen = 1ll << 30;  // positions (places of a sequence are counted in 32 bits)
// p = 2^(score - reference + kShift), and a reference moves when a score exceeds it by
// 2^kMove. fp16: p up to 2^15, and small ones keep their bits (bf16 has fp32's range).
template <bool kBf16>
constexpr float kShift = kBf16 ? 0.0f : 11.0f;
template <bool kBf16>
constexpr float kMove = kBf16 ? 8.0f : 4.0f;

// Workspace: for each CTA the unit that begins in it and goes on in others
// (batch index, unit, last CTA; last CTA -1: none), then two partial results per
// CTA (of a unit that began before it, of one that goes on behind it): 16
// maxima, 16 sums, 16 x 128 values.
constexpr int kPartFloats = 32 + 16 * 128;
constexpr size_t kWsBytes = kMaxGrid * (sizeof(int4) + 2 * kPartFloats * sizeof(float));

template <bool kBf16>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if (kBf16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// A shared-memory load that stays where it is (not hoisted out of a loop).
__device__ __forceinline__ uint4 reload16(const uint4* p) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem_u32(p)));
  return v;
}

__device__ __forceinline__ void st_shared_cluster_v4(uint32_t a, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// p of two heads as `kParts` pairs of 16-bit values (p0 in the low halves) whose sums
// they are: cut off towards 0, the last of fp16 rounded. Where p > 0 all of them are: 0 would
// make NaN of an infinite value in V, and so would values of both signs. The least value
// instead of 0 adds to p no more than 2^-126 in bf16, and in fp16 2^-23 where p is below
// 2^-11 of the weight at the reference (2^-34 of that weight).
template <bool kBf16>
constexpr int kParts = kBf16 ? 3 : 2;

__device__ __forceinline__ uint32_t cut_bf16x2(float p0, float p1) {
  return __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
}

template <bool kBf16>
__device__ __forceinline__ void split2(float p0, float p1, uint32_t (&w)[kParts<kBf16>]) {
  const uint32_t top = cut_bf16x2(p0, p1);
  if constexpr (kBf16) {
    const uint32_t least = __vminu2(top, 0x00800080u);  // 2^-126, or 0
    w[0] = top;
#pragma unroll
    for (int i = 1; i < kParts<kBf16>; ++i) {
      p0 -= __uint_as_float(__float_as_uint(p0) & 0xFFFF0000u);
      p1 -= __uint_as_float(__float_as_uint(p1) & 0xFFFF0000u);
      w[i] = __vmaxu2(cut_bf16x2(p0, p1), least);
    }
  } else {
    const uint32_t least = __vminu2(top, 0x00010001u);  // 2^-24, or 0
    uint32_t hi;
    asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(p1), "f"(p0));
    const float2 back = unpack2<false>(hi);
    w[0] = __vmaxu2(hi, least);
    w[1] = __vmaxu2(pack2<false>(p0 - back.x, p1 - back.y), least);
  }
}

// Output of head h (dimensions d .. d + 3) and its logarithm of the sum, from
// the reference maximum, the sum and the values against it.
template <bool kBf16>
__device__ __forceinline__ void write_out(const PagedAttnArgs& a, int b, int h, int d, float m, float sum, float4 v) {
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint2 w;
  w.x = pack2<kBf16>(v.x * inv, v.y * inv);
  w.y = pack2<kBf16>(v.z * inv, v.w * inv);
  if (sum == 0.0f) w = make_uint2(0u, 0u);  // (0 times an infinite value was NaN)
  *reinterpret_cast<uint2*>(a.o + b * a.ldo + static_cast<long long>(h) * a.kv.dh + d) = w;
  if (d == 0 && a.lse)
    a.lse[static_cast<long long>(b) * a.H + h] = sum == 0.0f ? -INFINITY : (m - kShift<kBf16>) * 0.6931471805599453f + logf(sum);
}

// How the tiles of all units in one row are dealt: CTA c has q of them from
// c q + min(c, r), one more if c < r.
struct Plan {
  unsigned long long q, r;
  unsigned long long first;  // this CTA's
  unsigned long long at;     // the tiles of the sequences before b
  int b;                     // the sequence that `first` lies in
  int pieces;                // 1: a CTA for each kMinTiles of a unit; 0: equal ranges
};

// The places of a unit in that row: its tiles and then what it costs beside them
// (without which CTAs of many short units finished last: 24 sequences of up to
// 2048 x 40 heads 118 us), or its tiles rounded up to whole pieces.
__device__ __forceinline__ int span_of(int tiles, int pieces) {
  return pieces ? (tiles + kMinTiles - 1) / kMinTiles * kMinTiles : tiles + kUnitCost;
}

// 64-bit quotients of numbers that mostly fit in 32.
__device__ __forceinline__ unsigned long long quotient(unsigned long long a, unsigned long long b) {
  if (((a | b) >> 32) == 0) return static_cast<unsigned int>(a) / static_cast<unsigned int>(b);
  return a / b;
}

template <bool kBf16, int kDh, int kNt, bool kSmallPage, bool kCluster>
__global__ void __launch_bounds__(kThreads, kNt == 1 ? 3 : 2) paged_attention_kernel(const PagedAttnArgs a) {
  constexpr int kHeads = 8 * kNt;
  constexpr int kRep = 128 / kDh;          // blocks of 16 positions per warp and tile: 8 KB of keys and values
  constexpr int kTile = 16 * kRep * kWarps;
  constexpr int kKc = kDh / 32;            // 16-byte pieces of a key row per lane
  constexpr int kVc = kDh / 64;            // of a value row
  extern __shared__ __align__(16) float so[];  // [kWarps][kHeads][kDh]
  __shared__ float sm[kWarps][kHeads], sl[kWarps][kHeads];
  __shared__ uint4 sq[kWarps][kNt][kKc][32];  // the query operand, lane by lane (the registers are for the loads)
  __shared__ unsigned long long scan[2][kWarps];
  __shared__ Plan plan;

  const PagedCache& c = a.kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int group = a.H / c.Hkv, parts = (group + kHeads - 1) / kHeads, units = c.Hkv * parts;
  const long long room = min(static_cast<long long>(c.table_cols) << c.page_log2, kMaxLen);
  const float c2 = a.scale * 1.4426950408889634f;
  int4* split = static_cast<int4*>(a.ws);
  float* partial = reinterpret_cast<float*>(split + kMaxGrid);

  if (kCluster) cluster_begun_arrive();
  pdl_wait();
  pdl_launch_dependents();

  auto length = [&](int b) -> int {
    const int n = a.lens[b];
    return n < 0 ? 0 : n > room ? static_cast<int>(room) : n;
  };
  auto tiles_of = [&](int n) { return n <= kTile ? 1 : (n + kTile - 1) / kTile; };

  unsigned long long x = 0, last = 1;
  int b, u, tile = 0;
  const int cs = kCluster ? static_cast<int>(cluster_nctarank()) : 1, rank = kCluster ? static_cast<int>(cluster_ctarank()) : 0;
  if (kCluster) {
    const int unit = static_cast<int>(blockIdx.x) / cs;
    b = unit / units;
    u = unit % units;
    if (a.lens[b] > room && rank == 0 && u == 0 && tid == 0) atomicOr(&g_paged_err, kErrIndex);
  } else {
    // The tiles before this thread's sequences, their sum, and from these the
    // CTA's range and where it begins. Few tiles: a CTA for each kMinTiles of a
    // unit, so that none has two units one after the other; else equal ranges.
    typedef unsigned long long u64;
    const int per = (c.seqs + kThreads - 1) / kThreads, b0 = min(c.seqs, tid * per), b1 = min(c.seqs, b0 + per);
    u64 mine = 0, padded = 0;
    for (int i = b0; i < b1; ++i) {
      const int n = tiles_of(length(i));
      if (a.lens[i] > room && blockIdx.x == 0) atomicOr(&g_paged_err, kErrIndex);
      mine += span_of(n, 0);
      padded += span_of(n, 1);
    }
    u64 upto = mine, upto_p = padded;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const u64 v = __shfl_up_sync(0xFFFFFFFFu, upto, d), w = __shfl_up_sync(0xFFFFFFFFu, upto_p, d);
      if (lane >= d) {
        upto += v;
        upto_p += w;
      }
    }
    if (lane == 31) {
      scan[0][warp] = upto;
      scan[1][warp] = upto_p;
    }
    __syncthreads();
    u64 all = 0, all_p = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) {
        upto += scan[0][w];
        upto_p += scan[1][w];
      }
      all += scan[0][w];
      all_p += scan[1][w];
    }
    const bool pieces = all_p * units <= static_cast<u64>(gridDim.x) * kMinTiles;
    const u64 total = (pieces ? all_p : all) * units, cta = blockIdx.x;
    if (pieces) {
      upto = upto_p;
      mine = padded;
    }
    const u64 q = pieces ? kMinTiles : quotient(total, gridDim.x), r = pieces ? 0 : total - q * gridDim.x;
    const u64 first = cta * q + min(cta, r);
    if (tid == 0) split[blockIdx.x] = make_int4(0, 0, -1, 0);
    if (first >= total) return;  // (the whole CTA)
    if (first >= (upto - mine) * units && first < upto * units) {
      u64 at = (upto - mine) * units;
      for (int i = b0; i < b1; ++i) {
        const u64 n = static_cast<u64>(span_of(tiles_of(length(i)), pieces)) * units;
        if (first < at + n) {
          plan.b = i;
          break;
        }
        at += n;
      }
      plan.q = q;
      plan.r = r;
      plan.first = first;
      plan.at = at;
      plan.pieces = pieces;
    }
    __syncthreads();
    x = plan.first;
    last = x + plan.q + (blockIdx.x < plan.r ? 1 : 0);
    b = plan.b;
    const int span = span_of(tiles_of(length(b)), plan.pieces);
    u = static_cast<int>(quotient(x - plan.at, span));
    tile = static_cast<int>(x - plan.at - static_cast<unsigned long long>(u) * span);
  }
  while (x < last && b < c.seqs) {
    const int len = length(b), tiles = tiles_of(len);
    int stop, tile_end;
    if (kCluster) {  // the CTA's share of the unit (none: a part of no weight)
      tile = rank * tiles / cs;
      stop = tile_end = (rank + 1) * tiles / cs;
    } else {
      stop = static_cast<int>(min(static_cast<unsigned long long>(span_of(tiles, plan.pieces)), tile + (last - x)));
      tile_end = min(tiles, stop);
    }
    auto next_unit = [&]() {
      x += stop - tile;
      tile = 0;
      if (++u == units) {
        u = 0;
        ++b;
      }
    };
    if (!kCluster && tile >= tile_end) {  // none of its tiles are in the range
      next_unit();
      continue;
    }
    const int hk = u / parts, h0 = hk * group + (u % parts) * kHeads;
    const int heads = min(kHeads, hk * group + group - h0);
    const int32_t* table = c.table + static_cast<long long>(b) * c.table_ld;
    const uint16_t* kh = c.k + hk * c.head_stride + t * 8;
    const uint16_t* vh = c.v + hk * c.head_stride + g * 8;
    const int slots = (1 << c.page_log2) - 1;

    // Element offset of position j in the cache (without the head), -1 if it is not to be read.
    auto offset = [&](int j) -> long long {
      if (j >= len) return -1;
      const int page = table[j >> c.page_log2];
      if (static_cast<unsigned int>(page) >= static_cast<unsigned int>(c.pages)) {
        atomicOr(&g_paged_err, kErrIndex);
        return -1;
      }
      return page * c.page_stride + (j & slots) * c.token_stride;
    };

    float o[kNt][kVc][4][4];  // O^T: [.][hh][j]: dimensions 64 hh + 8 g + 2 j (+ 1), heads 2 t, 2 t + 1
    float ref[kNt][2], l[kNt][2];
#pragma unroll
    for (int n = 0; n < kNt; ++n) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ref[n][e] = -INFINITY;
        l[n][e] = 0.0f;
      }
#pragma unroll
      for (int hh = 0; hh < kVc; ++hh)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[n][hh][j][e] = 0.0f;
    }

    uint4 kr[kRep][kKc][2], vr[kRep][kVc][4];
    // With pages of 16 and more a block of 16 positions lies in one page: its
    // offset is looked up a tile ahead of its loads, and its rows past the
    // length are read too (they are the page's) but do not count. With smaller
    // pages each row has an offset.
    constexpr int kLook = kSmallPage ? 6 : 1;
    long long off[kRep][kLook];
    auto look = [&](int tl) {
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        const int j = tl * kTile + (warp * kRep + r) * 16;
        if (kSmallPage) {
          off[r][0] = offset(j + g);
          off[r][1] = offset(j + g + 8);
          off[r][2] = offset(j + 2 * t);
          off[r][3] = offset(j + 2 * t + 1);
          off[r][4] = offset(j + 2 * t + 8);
          off[r][5] = offset(j + 2 * t + 9);
        } else {
          off[r][0] = offset(j);
        }
      }
    };
    // The keys of rows g, g + 8 of block r that count: bits 2 r, 2 r + 1 (of
    // the loaded keys: live).
    uint32_t live = 0;
    auto load_k = [&](int tl) {
      live = 0;
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        const int j = tl * kTile + (warp * kRep + r) * 16;
        if (kSmallPage) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bool valid = off[r][e] >= 0;
            live |= valid ? 1u << (2 * r + e) : 0u;
#pragma unroll
            for (int i = 0; i < kKc; ++i) {
              kr[r][i][e] = make_uint4(0u, 0u, 0u, 0u);
              if (valid) kr[r][i][e] = ldg_stream16(kh + off[r][e] + 32 * i);
            }
          }
        } else if (off[r][0] >= 0) {
          live |= (j + g < len ? 1u << (2 * r) : 0u) | (j + g + 8 < len ? 2u << (2 * r) : 0u);
          const uint16_t* p = kh + off[r][0] + g * c.token_stride;
#pragma unroll
          for (int i = 0; i < kKc; ++i) kr[r][i][0] = ldg_stream16(p + 32 * i);
          p += 8 * c.token_stride;
#pragma unroll
          for (int i = 0; i < kKc; ++i) kr[r][i][1] = ldg_stream16(p + 32 * i);
        }
      }
    };
    auto load_v = [&](int tl) {
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        if (kSmallPage) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int hh = 0; hh < kVc; ++hh) {
              vr[r][hh][e] = make_uint4(0u, 0u, 0u, 0u);
              if (off[r][2 + e] >= 0) vr[r][hh][e] = ldg_stream16(vh + off[r][2 + e] + 64 * hh);
            }
        } else if (off[r][0] >= 0) {
          const uint16_t* p = vh + off[r][0] + 2 * t * c.token_stride;
#pragma unroll
          for (int e = 0; e < 4; ++e) {  // rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
            for (int hh = 0; hh < kVc; ++hh) vr[r][hh][e] = ldg_stream16(p + 64 * hh);
            p += (e == 1 ? 7 : 1) * c.token_stride;
          }
        }
      }
    };

    if (!kCluster || tile < tile_end) look(tile);
    // Q: head g of each 8, dimensions 32 i + 8 t .. (on its way beside the page numbers)
    uint4 q[kNt][kKc];
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int i = 0; i < kKc; ++i) {
        const int h = 8 * n + g;
        q[n][i] = make_uint4(0u, 0u, 0u, 0u);
        if (h < heads) q[n][i] = *reinterpret_cast<const uint4*>(a.q + b * a.ldq + static_cast<long long>(h0 + h) * kDh + 32 * i + 8 * t);
      }
    if (!kCluster || tile < tile_end) {
      load_k(tile);
      load_v(tile);
      look(tile + 1);
    }
    __syncwarp();
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int i = 0; i < kKc; ++i) sq[warp][n][i][lane] = q[n][i];
    __syncwarp();
    for (int tl = tile; tl < tile_end; ++tl) {
      const bool more = tl + 1 < tile_end;
      float s[kRep][kNt][4];
#pragma unroll
      for (int r = 0; r < kRep; ++r)
#pragma unroll
        for (int n = 0; n < kNt; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r][n][e] = 0.0f;
#pragma unroll
          for (int i = 0; i < kKc; ++i) {
            const uint4 f = reload16(&sq[warp][n][i][lane]);
            mma16816<kBf16>(s[r][n], kr[r][i][0].x, kr[r][i][1].x, kr[r][i][0].y, kr[r][i][1].y, f.x, f.y);
            mma16816<kBf16>(s[r][n], kr[r][i][0].z, kr[r][i][1].z, kr[r][i][0].w, kr[r][i][1].w, f.z, f.w);
          }
        }
      const uint32_t counts = live;
      if (more) load_k(tl + 1);
      // scores in powers of two; positions that do not count have none
#pragma unroll
      for (int r = 0; r < kRep; ++r)
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r][n][e] *= c2;
      constexpr uint32_t kAll = (1u << (2 * kRep)) - 1u;
      if (!__all_sync(0xFFFFFFFFu, counts == kAll)) {
#pragma unroll
        for (int r = 0; r < kRep; ++r) {
#pragma unroll
          for (int n = 0; n < kNt; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(counts >> (2 * r + (e >> 1)) & 1u)) s[r][n][e] = -INFINITY;
          // values of these positions may be anything: 0 (p is 0, but 0 times infinity is not)
          const uint32_t rows = __ballot_sync(0xFFFFFFFFu, t == 0 && (counts >> (2 * r) & 1u)) |
                                __ballot_sync(0xFFFFFFFFu, t == 0 && (counts >> (2 * r) & 2u)) << 1;  // row i: bit 4 i, 4 (i - 8) + 1
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(rows >> (4 * (2 * t + (e & 1)) + (e >> 1)) & 1u)) {
#pragma unroll
              for (int hh = 0; hh < kVc; ++hh) vr[r][hh][e] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
      }
      bool move = false;
#pragma unroll
      for (int r = 0; r < kRep; ++r)
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) move = move || s[r][n][e] > ref[n][e & 1] + kMove<kBf16>;
      if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = ref[n][e];
#pragma unroll
            for (int r = 0; r < kRep; ++r) m = fmaxf(m, fmaxf(s[r][n][e], s[r][n][e + 2]));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
            const float alpha = m == ref[n][e] ? 1.0f : exp2_fast(ref[n][e] - m);
            ref[n][e] = m;
            l[n][e] *= alpha;
#pragma unroll
            for (int hh = 0; hh < kVc; ++hh)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                o[n][hh][j][e] *= alpha;
                o[n][hh][j][e + 2] *= alpha;
              }
          }
      }
      float from[kNt][2];  // (no score of the head yet: those there are are -inf, or NaN)
#pragma unroll
      for (int n = 0; n < kNt; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) from[n][e] = ref[n][e] == -INFINITY ? 0.0f : ref[n][e] - kShift<kBf16>;
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        uint32_t pw[kNt][kParts<kBf16>][2];
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {  // rows g, g + 8
            const float p0 = exp2_fast(s[r][n][2 * e] - from[n][0]), p1 = exp2_fast(s[r][n][2 * e + 1] - from[n][1]);
            l[n][0] += p0;
            l[n][1] += p1;
            uint32_t w[kParts<kBf16>];
            split2<kBf16>(p0, p1, w);
#pragma unroll
            for (int i = 0; i < kParts<kBf16>; ++i) pw[n][i][e] = transpose8x8(w[i]);
          }
#pragma unroll
        for (int hh = 0; hh < kVc; ++hh) {
          const uint4* w = vr[r][hh];
          const uint32_t w0[4] = {w[0].x, w[0].y, w[0].z, w[0].w}, w1[4] = {w[1].x, w[1].y, w[1].z, w[1].w};
          const uint32_t w2[4] = {w[2].x, w[2].y, w[2].z, w[2].w}, w3[4] = {w[3].x, w[3].y, w[3].z, w[3].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t a0 = __byte_perm(w0[j], w1[j], 0x5410), a1 = __byte_perm(w0[j], w1[j], 0x7632);
            const uint32_t a2 = __byte_perm(w2[j], w3[j], 0x5410), a3 = __byte_perm(w2[j], w3[j], 0x7632);
#pragma unroll
            for (int n = 0; n < kNt; ++n)
#pragma unroll
              for (int i = 0; i < kParts<kBf16>; ++i) mma16816<kBf16>(o[n][hh][j], a0, a1, a2, a3, pw[n][i][0], pw[n][i][1]);
          }
        }
      }
      if (more) {
        load_v(tl + 1);
        look(tl + 2);
      }
    }

    // The warps' parts into shared memory.
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int h = 8 * n + 2 * t + e;
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, l[n][e], d);
        if (g == 0) {
          sm[warp][h] = ref[n][e];
          sl[warp][h] = l[n][e];
        }
        if (h < heads) {
#pragma unroll
          for (int hh = 0; hh < kVc; ++hh) {
            float* d = so + (warp * kHeads + h) * kDh + 64 * hh + 8 * g;
#pragma unroll
            for (int j = 0; j < 4; j += 2)
              *reinterpret_cast<float4*>(d + 2 * j) = make_float4(o[n][hh][j][e], o[n][hh][j][e + 2],
                                                                  o[n][hh][j + 1][e], o[n][hh][j + 1][e + 2]);
          }
        }
      }
    __syncthreads();

    // Their maxima, sums and values added up, to done(head, dimension, maximum, sum, four values).
    auto add_warps = [&](auto&& done) {
      for (int i = tid; i < heads * (kDh / 4); i += kThreads) {
        const int h = i / (kDh / 4), d = (i % (kDh / 4)) * 4;
        float m = sm[0][h], sum = 0.0f;
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm[w][h]);
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = sm[w][h] == -INFINITY ? 0.0f : exp2_fast(sm[w][h] - m);
          const float4 z = *reinterpret_cast<const float4*>(so + (w * kHeads + h) * kDh + d);
          sum += sl[w][h] * f;
          v.x += z.x * f;
          v.y += z.y * f;
          v.z += z.z * f;
          v.w += z.w * f;
        }
        done(h, d, m, sum, v);
      }
    };
    if (kCluster) {  // the CTAs' parts to the first of them, and their sum there
      constexpr int kPart = kHeads * kDh + 2 * kHeads;
      float* const all = so + kWarps * kHeads * kDh;  // [cs][kPart]
      cluster_begun_wait();
      add_warps([&](int h, int d, float m, float sum, float4 v) {
        const uint32_t at = mapa_shared(smem_u32(all + rank * kPart), 0);
        st_shared_cluster_v4(at + 4 * (h * kDh + d), v);
        if (d == 0) {
          st_shared_cluster_u32(at + 4 * (kHeads * kDh + h), __float_as_uint(m));
          st_shared_cluster_u32(at + 4 * (kHeads * kDh + kHeads + h), __float_as_uint(sum));
        }
      });
      cluster_sync();
      if (rank != 0) return;
      for (int i = tid; i < heads * (kDh / 4); i += kThreads) {
        const int h = i / (kDh / 4), d = (i % (kDh / 4)) * 4;
        float m = -INFINITY, sum = 0.0f;
        for (int r = 0; r < cs; ++r) m = fmaxf(m, all[r * kPart + kHeads * kDh + h]);
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int r = 0; r < cs; ++r) {
          const float* const part = all + r * kPart;
          const float mr = part[kHeads * kDh + h], f = mr == -INFINITY ? 0.0f : exp2_fast(mr - m);
          const float4 z = *reinterpret_cast<const float4*>(part + h * kDh + d);
          sum += part[kHeads * kDh + kHeads + h] * f;
          v.x += z.x * f;
          v.y += z.y * f;
          v.z += z.z * f;
          v.w += z.w * f;
        }
        write_out<kBf16>(a, b, h0 + h, d, m, sum, v);
      }
      return;
    }
    if (tile == 0 && tile_end == tiles) {
      add_warps([&](int h, int d, float m, float sum, float4 v) { write_out<kBf16>(a, b, h0 + h, d, m, sum, v); });
    } else {
      float* part = partial + static_cast<size_t>(2 * blockIdx.x + (tile == 0 ? 1 : 0)) * kPartFloats;
      add_warps([&](int h, int d, float m, float sum, float4 v) {
        if (d == 0) {
          part[h] = m;
          part[16 + h] = sum;
        }
        *reinterpret_cast<float4*>(part + 32 + h * kDh + d) = v;
      });
      if (tile == 0 && tid == 0) {  // who else has parts of the unit
        const unsigned long long y = x + tiles - 1, more = plan.r * (plan.q + 1);
        split[blockIdx.x] =
            make_int4(b, u, static_cast<int>(y < more ? quotient(y, plan.q + 1) : plan.r + quotient(y - more, plan.q)), 0);
      }
    }
    __syncthreads();  // the shared results have been read

    next_unit();
  }
}

// Joins the units that several CTAs share: CTA (x, y) head y of the unit that
// begins in CTA x of the kernel before, from that one's part and those of the
// following. Each warp takes every fourth part, kBatch at a time with their loads
// in flight together (76 parts of 4 heads one after the other took 15 us; a CTA of
// 16 warps for 4 heads 1.5 us more than this for 57).
constexpr int kJoinWarps = 4;

template <bool kBf16, int kDh, int kNt>
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const PagedAttnArgs a) {
  constexpr int kHeads = 8 * kNt, kBatch = 16, kJd = kDh / 32;  // parts; dimensions per lane
  __shared__ __align__(16) float so[kJoinWarps][kDh];
  __shared__ float sm[kJoinWarps], sl[kJoinWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = a.H / a.kv.Hkv, parts = (group + kHeads - 1) / kHeads;
  pdl_wait();
  pdl_launch_dependents();
  const int4* split = static_cast<const int4*>(a.ws);
  const float* partial = reinterpret_cast<const float*>(split + kMaxGrid);
  const int c0 = static_cast<int>(blockIdx.x), h = static_cast<int>(blockIdx.y);
  // A warp's first part beside the description, which says whether it is one (most units have few)
  const int c_first = min(c0 + warp, kMaxGrid - 1);
  const float* p0 = partial + static_cast<size_t>(2 * c_first + (warp == 0)) * kPartFloats;
  const float m0 = p0[h], l0 = p0[16 + h];
  float z0[kJd];
#pragma unroll
  for (int e = 0; e < kJd; e += 2) {
    const float2 v = *reinterpret_cast<const float2*>(p0 + 32 + h * kDh + lane * kJd + e);
    z0[e] = v.x;
    z0[e + 1] = v.y;
  }
  const int4 unit = split[blockIdx.x];
  const int c1 = unit.z;
  if (c1 < 0) return;
  const int hk = unit.y / parts, h0 = hk * group + (unit.y % parts) * kHeads;
  if (h >= hk * group + group - h0) return;
  float jm = -INFINITY, jl = 0.0f, jo[kJd];
#pragma unroll
  for (int e = 0; e < kJd; ++e) jo[e] = 0.0f;
  if (c0 + warp <= c1) {
    jm = m0;
    jl = l0;
#pragma unroll
    for (int e = 0; e < kJd; ++e) jo[e] = z0[e];
  }
  for (int k0 = c0 + warp + kJoinWarps; k0 <= c1; k0 += kBatch * kJoinWarps) {
    float mk[kBatch], lk[kBatch], z[kBatch][kJd];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int cta = k0 + i * kJoinWarps;
      const float* p = partial + static_cast<size_t>(2 * cta) * kPartFloats;
      mk[i] = -INFINITY;
      lk[i] = 0.0f;
#pragma unroll
      for (int e = 0; e < kJd; ++e) z[i][e] = 0.0f;
      if (cta <= c1) {
        mk[i] = p[h];
        lk[i] = p[16 + h];
        if (kJd == 4) {
          const float4 v = *(reinterpret_cast<const float4*>(p + 32 + h * kDh) + lane);
          z[i][0] = v.x;
          z[i][1] = v.y;
          z[i][2 % kJd] = v.z;
          z[i][3 % kJd] = v.w;
        } else {
          const float2 v = *(reinterpret_cast<const float2*>(p + 32 + h * kDh) + lane);
          z[i][0] = v.x;
          z[i][1] = v.y;
        }
      }
    }
    float m = jm;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) m = fmaxf(m, mk[i]);
    const float of = jm == -INFINITY ? 0.0f : exp2_fast(jm - m);
    jm = m;
    jl *= of;
#pragma unroll
    for (int e = 0; e < kJd; ++e) jo[e] *= of;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float f = mk[i] == -INFINITY ? 0.0f : exp2_fast(mk[i] - m);
      jl += lk[i] * f;
#pragma unroll
      for (int e = 0; e < kJd; ++e) jo[e] += z[i][e] * f;
    }
  }
  if (lane == 0) {
    sm[warp] = jm;
    sl[warp] = jl;
  }
#pragma unroll
  for (int e = 0; e < kJd; ++e) so[warp][lane * kJd + e] = jo[e];
  __syncthreads();
  const int d = static_cast<int>(threadIdx.x) * 4;
  if (d >= kDh) return;
  float m = sm[0], sum = 0.0f;
#pragma unroll
  for (int w = 1; w < kJoinWarps; ++w) m = fmaxf(m, sm[w]);
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) {
    const float f = sm[w] == -INFINITY ? 0.0f : exp2_fast(sm[w] - m);
    const float4 z = *reinterpret_cast<const float4*>(&so[w][d]);
    sum += sl[w] * f;
    v.x += z.x * f;
    v.y += z.y * f;
    v.z += z.z * f;
    v.w += z.w * f;
  }
  write_out<kBf16>(a, unit.x, h0 + h, d, m, sum, v);
}

template <int kDh, int kNt>
constexpr size_t cluster_smem(int cs) {
  return (static_cast<size_t>(kWarps + cs) * 8 * kNt * kDh + static_cast<size_t>(cs) * 2 * 8 * kNt) * sizeof(float);
}

struct ClusterLaunch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  ClusterLaunch(int units, int cs, size_t smem, cudaStream_t stream) {
    cfg.gridDim = dim3(static_cast<unsigned>(units * cs));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cs);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
};

// The shared memory that a cluster's CTAs ask for, whatever their number.
template <bool kBf16, int kDh, int kNt, bool kSmallPage>
cudaError_t allow_clusters() {
  static SmemLimit limit;
  return limit.allow(paged_attention_kernel<kBf16, kDh, kNt, kSmallPage, true>, cluster_smem<kDh, kNt>(kMaxCluster));
}

// Clusters of cs CTAs that the GPU holds at once; 0 where it does not say.
template <bool kBf16, int kDh, int kNt, bool kSmallPage>
int clusters_at_once(int cs) {
  static DeviceNumber known[kMaxCluster + 1];
  int n = 0;
  const cudaError_t e = known[cs].get(&n, [cs](int* number) {
    const cudaError_t le = allow_clusters<kBf16, kDh, kNt, kSmallPage>();
    if (le != cudaSuccess) return le;
    ClusterLaunch l(1, cs, cluster_smem<kDh, kNt>(cs), nullptr);
    l.cfg.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(number, paged_attention_kernel<kBf16, kDh, kNt, kSmallPage, true>, &l.cfg);
  });
  if (e == cudaSuccess) return n;
  cudaGetLastError();
  return 0;
}

// A cluster of cs CTAs for each unit.
template <bool kBf16, int kDh, int kNt, bool kSmallPage>
cudaError_t launch_clusters(const PagedAttnArgs& a, int units, int cs, cudaStream_t stream, unsigned int* launches) {
  cudaError_t e = allow_clusters<kBf16, kDh, kNt, kSmallPage>();
  if (e != cudaSuccess) return e;
  const ClusterLaunch l(units, cs, cluster_smem<kDh, kNt>(cs), stream);
  e = cudaLaunchKernelEx(&l.cfg, paged_attention_kernel<kBf16, kDh, kNt, kSmallPage, true>, a);
  if (e == cudaSuccess) ++*launches;
  return e;
}

template <bool kBf16, int kDh, int kNt, bool kSmallPage>
cudaError_t launch(const PagedAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  constexpr size_t smem = static_cast<size_t>(kWarps) * 8 * kNt * kDh * sizeof(float);
  static SmemLimit limit;
  auto* kernel = paged_attention_kernel<kBf16, kDh, kNt, kSmallPage, false>;
  const cudaError_t le = limit.allow(kernel, smem);
  if (le != cudaSuccess) return le;
  // CTAs for every tile that the table has room for, at most a wave
  const int group = a.H / a.kv.Hkv;
  const long long units = static_cast<long long>(a.kv.Hkv) * ((group + 8 * kNt - 1) / (8 * kNt)) * a.kv.seqs;
  constexpr int kTile = 16 * (128 / kDh) * kWarps;
  const long long room = std::max(1ll, ((static_cast<long long>(a.kv.table_cols) << a.kv.page_log2) + kTile - 1) / kTile);
  const int wave = std::min(kMaxGrid, num_sms() * (kNt == 1 ? 3 : 2));
  // A cluster for each unit, if all have room at once (an eighth is left over: behind another kernel's last
  // CTAs 144 clusters of 3 took 23 us, of 2 17.7) and none of its CTAs has so many tiles more than equal ranges give
  // it, of sequences a third as long as the table, that the second kernel costs less. The table's width stands for the
  // lengths here, which the host does not know: 704 positions x 40 heads take 6.2 us in tables of up to 4096, 9.4 in
  // wider ones (8 heads 4.7, 8.7). us, with it and without: one sequence of 704 x 40 heads 6.2, 9.4, of 2048 x 8 6.5, 9.0, of 4096 x 8 11.0, 10.7, half as long as the table 4.1,
  // 7.9; 16 of up to 768 x 8 10.3, 13.7, 12 of up to 768 x 32 (12 tiles) 21.2, 19.6. A CTA for each of up to twice as many units of few tiles: 25 of 128 x 32
  // 14.2, 15.9, of 256 22.0, 23.5 (of five waves: 100 of 200 x 32 73, 66).
  if (units <= wave || (units <= 2 * wave && room <= 2 * kMinTiles)) {
    const bool spread = units * room <= num_sms();  // a tile each (256 x 32 heads 3.9, of two 4.8; 4 of 512 x 8 5.5, 4.9)
    int cs = static_cast<int>(std::min<long long>(kMaxCluster, spread ? room : (room + kMinTiles - 1) / kMinTiles));
    while (cs > 1 && units * 8 > clusters_at_once<kBf16, kDh, kNt, kSmallPage>(cs) * 7) --cs;
    if ((room + cs - 1) / cs <= units * room / (3 * wave) + kJoinTiles)
      return launch_clusters<kBf16, kDh, kNt, kSmallPage>(a, static_cast<int>(units), cs, stream, launches);
  }
  const int grid = room >= wave || units >= wave ? wave : static_cast<int>(std::min<long long>(wave, units * room));
  cudaError_t e = launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads), smem, stream, a);
  if (e != cudaSuccess) return e;
  ++*launches;
  const unsigned heads = static_cast<unsigned>(std::min(group, 8 * kNt));
  e = launch_pdl(join_kernel<kBf16, kDh, kNt>, dim3(static_cast<unsigned>(grid), heads), dim3(32 * kJoinWarps), 0, stream,
                 a);
  if (e == cudaSuccess) ++*launches;
  return e;
}

template <bool kBf16, int kDh>
cudaError_t launch_for(const PagedAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  const bool wide = a.H / a.kv.Hkv > 8, small = a.kv.page_log2 < 4;
  if (wide) return small ? launch<kBf16, kDh, 2, true>(a, stream, launches) : launch<kBf16, kDh, 2, false>(a, stream, launches);
  return small ? launch<kBf16, kDh, 1, true>(a, stream, launches) : launch<kBf16, kDh, 1, false>(a, stream, launches);
}

}  // namespace

size_t paged_attention_workspace_bytes() { return kWsBytes; }

cudaError_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  if (a.kv.bf16) return a.kv.dh == 64 ? launch_for<true, 64>(a, stream, launches) : launch_for<true, 128>(a, stream, launches);
  return a.kv.dh == 64 ? launch_for<false, 64>(a, stream, launches) : launch_for<false, 128>(a, stream, launches);
}

unsigned int paged_read_and_clear_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_paged_err, sizeof(v));
  cudaMemcpyToSymbol(g_paged_err, &z, sizeof(z));
  return v;
}

}  // namespace p4q
