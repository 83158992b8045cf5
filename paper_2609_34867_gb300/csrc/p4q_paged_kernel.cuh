// The attention of one new token per sequence over a paged cache, for whatever C says how
// to go through its tiles: 16-bit keys and values, codes, the positions behind a prefix.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>

#include "p4q_paged.cuh"
#include "p4q_paged_prefix.cuh"

namespace p4q {
namespace {

using namespace paged;

constexpr int kMaxGrid = 640;    // CTAs of a launch at most (partial results of the workspace)
constexpr int kMinTiles = 2;     // tiles per CTA at least, of one unit
constexpr int kUnitCost = 2;     // what a unit costs beside its tiles, in tiles
constexpr int kMaxCluster = 8;   // CTAs that share a unit as a cluster
constexpr int kJoinTiles = 8;    // what the second kernel costs, in tiles of a CTA
constexpr long long kMaxLen = 1ll << 30;  // positions (places of a sequence are counted in 32 bits)

// Workspace: for each CTA the unit that begins in it and goes on in others
// (batch index, unit, last CTA; last CTA -1: none), then two partial results per
// CTA (of a unit that began before it, of one that goes on behind it): 16
// maxima, 16 sums, 16 x 128 values.
constexpr int kPartFloats = 32 + 16 * 128;
constexpr size_t kWsBytes = kMaxGrid * (sizeof(int4) + 2 * kPartFloats * sizeof(float));

__device__ __forceinline__ void st_shared_cluster_v4(uint32_t a, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// Output of head h (dimensions d .. d + 3) and its logarithm of the sum, from
// the reference maximum, the sum and the values against it.
template <class C>
__device__ __forceinline__ void write_out(const typename C::Args& a, int b, int h, int d, float m, float sum, float4 v) {
  if constexpr (C::kOwnOnly) {  // a part of what another kernel adds up
    float* const part = a.own + (static_cast<long long>(b) * a.H + h) * (C::kDh + kPartExtra);
    *reinterpret_cast<float4*>(part + d) = v;
    if (d == 0) *reinterpret_cast<float4*>(part + C::kDh) = make_float4(m, sum, 0.0f, 0.0f);
    return;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint2 w;
  if (C::bf16(a))
    w = make_uint2(pack2<true>(v.x * inv, v.y * inv), pack2<true>(v.z * inv, v.w * inv));
  else
    w = make_uint2(pack2<false>(v.x * inv, v.y * inv), pack2<false>(v.z * inv, v.w * inv));
  if (sum == 0.0f) w = make_uint2(0u, 0u);  // (0 times an infinite value was NaN)
  *reinterpret_cast<uint2*>(a.o + b * a.ldo + static_cast<long long>(h) * C::kDh + d) = w;
  if (d == 0 && a.lse)
    a.lse[static_cast<long long>(b) * a.H + h] = sum == 0.0f ? -INFINITY : (m - C::kLift) * 0.6931471805599453f + logf(sum);
}

// How the tiles of all units in one row are dealt: CTA c has q of them from
// c q + min(c, r), one more if c < r.
struct Plan {
  unsigned long long q, r;
  unsigned long long first;  // this CTA's
  unsigned long long at;     // where the units of sequence b begin (kHeadsOuter: unit u of it)
  int u;                     // (kHeadsOuter)
  int b;                     // the sequence that `first` lies in
  int pieces;                // 1: a CTA for each kMinTiles of a unit; 0: equal ranges
};

// The places of a unit in that row: its tiles and then what it costs beside them
// (without which CTAs of many short units finished last: 24 sequences of up to
// 2048 x 40 heads 118 us), or its tiles rounded up to whole pieces.
__device__ __forceinline__ int span_of(int tiles, int pieces) {
  return pieces ? (tiles + kMinTiles - 1) / kMinTiles * kMinTiles : tiles + kUnitCost;
}

// The query heads of unit u of a sequence: count from h0. A unit is 8 NT of a key/value head's at most, or
// all of those of C::kSplit neighbouring ones, which its warps take turn by turn.
template <class C, int kNt>
struct UnitHeads {
  int h0, count;
  __device__ __forceinline__ UnitHeads(int u, int group, int parts) {
    const int hk = u / parts * C::kSplit;
    h0 = hk * group + u % parts * 8 * kNt;
    count = C::kSplit > 1 ? C::kSplit * group : min(8 * kNt, hk * group + group - h0);
  }
};

template <class C, int kNt, bool kCluster>
__global__ void __launch_bounds__(kThreads, C::ctas(kNt)) paged_attention_kernel(const typename C::Args a) {
  constexpr int kHeads = 8 * kNt;                  // of a warp
  constexpr int kUnitHeads = C::kSplit * kHeads;
  static_assert(kUnitHeads <= 16, "parts have room for 16 heads");
  constexpr int kDh = C::kDh, kVc = C::kVc, kTile = C::kTile;
  constexpr int kWarpFloats = C::warp_floats(kNt);
  extern __shared__ __align__(16) float so[];  // a warp's kWarpFloats: what it loads into, then its [kHeads][kDh] of O
  __shared__ float sm[kWarps][kHeads], sl[kWarps][kHeads];
  __shared__ uint4 sq[kWarps][kNt][kDh / 32][32];  // the query operand, lane by lane (the registers are for the loads)
  __shared__ unsigned long long scan[2][kWarps];
  __shared__ Plan plan;

  const auto& c = a.kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int group = a.H / c.Hkv, parts = (group + kHeads - 1) / kHeads, units = c.Hkv / C::kSplit * parts;
  const long long room = min(static_cast<long long>(c.table_cols) << c.page_log2, kMaxLen);
  int4* split = static_cast<int4*>(a.ws);
  float* partial = reinterpret_cast<float*>(split + kMaxGrid);

  if (kCluster) cluster_begun_arrive();
  if (C::kOwnOnly)
    see_earlier_kernels();
  else
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
    const u64 each = C::kHeadsOuter ? 1 : units;  // units of a sequence that lie side by side
    const int outer = C::kHeadsOuter ? static_cast<int>(quotient(first, total / units)) : 0;
    const u64 before = outer * (total / units);
    if (tid == 0) split[blockIdx.x] = make_int4(0, 0, -1, 0);
    if (first >= total) return;  // (the whole CTA)
    if (first - before >= (upto - mine) * each && first - before < upto * each) {
      u64 at = (upto - mine) * each + before;
      for (int i = b0; i < b1; ++i) {
        const u64 n = static_cast<u64>(span_of(tiles_of(length(i)), pieces)) * each;
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
      plan.u = outer;
    }
    __syncthreads();
    x = plan.first;
    last = x + plan.q + (blockIdx.x < plan.r ? 1 : 0);
    b = plan.b;
    const int span = span_of(tiles_of(length(b)), plan.pieces);
    const int at = C::kHeadsOuter ? 0 : static_cast<int>(quotient(x - plan.at, span));
    u = plan.u + at;
    tile = static_cast<int>(x - plan.at - static_cast<unsigned long long>(at) * span);
  }
  while (x < last && (C::kHeadsOuter ? u < units : b < c.seqs)) {
    const int len = length(b);
    const typename C::Behind behind(a, b, len);
    const int base = behind.from & ~15, tiles = tiles_of(len - base);  // (a block of 16 positions begins at one of the sequence's)
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
      if (C::kHeadsOuter) {
        if (++b == c.seqs) {
          b = 0;
          ++u;
        }
      } else if (++u == units) {
        u = 0;
        ++b;
      }
    };
    if (!kCluster && tile >= tile_end) {  // none of its tiles are in the range
      next_unit();
      continue;
    }
    const UnitHeads<C, kNt> uh(u, group, parts);
    const int h0 = uh.h0, hk = u / parts * C::kSplit + warp % C::kSplit;
    const int heads = C::kSplit > 1 ? group : uh.count;  // of the warp, from wh0
    const int wh0 = C::kSplit > 1 ? hk * group : h0;
    Part<kNt, kVc> acc;
    auto& o = acc.o;
    auto& ref = acc.ref;
    auto& l = acc.l;
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
    const Unit un = {c.table + static_cast<long long>(behind.row) * c.table_ld, b, hk, wh0, heads, len, behind.from, base};
    C::template attend<kNt>(a, un, tile, tile_end, sq[warp], so + warp * kWarpFloats, acc);

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
            float* d = so + warp * kWarpFloats + h * kDh + C::first_dim(hh, g);
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
      for (int i = tid; i < uh.count * (kDh / 4); i += kThreads) {
        const int hu = i / (kDh / 4), d = (i % (kDh / 4)) * 4;
        const int w0 = C::kSplit > 1 ? hu / group : 0, h = C::kSplit > 1 ? hu - w0 * group : hu;
        float m = sm[w0][h], sum = 0.0f;
#pragma unroll
        for (int w = w0 + C::kSplit; w < kWarps; w += C::kSplit) m = fmaxf(m, sm[w][h]);
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = w0; w < kWarps; w += C::kSplit) {
          const float f = sm[w][h] == -INFINITY ? 0.0f : exp2_fast(sm[w][h] - m);
          const float4 z = *reinterpret_cast<const float4*>(so + w * kWarpFloats + h * kDh + d);
          sum += sl[w][h] * f;
          v.x += z.x * f;
          v.y += z.y * f;
          v.z += z.z * f;
          v.w += z.w * f;
        }
        done(hu, d, m, sum, v);
      }
    };
    if (kCluster) {  // the CTAs' parts to the first of them, and their sum there
      constexpr int kPart = kUnitHeads * kDh + 2 * kUnitHeads;
      float* const all = so + kWarps * kWarpFloats;  // [cs][kPart]
      cluster_begun_wait();
      add_warps([&](int h, int d, float m, float sum, float4 v) {
        const uint32_t at = mapa_shared(smem_u32(all + rank * kPart), 0);
        st_shared_cluster_v4(at + 4 * (h * kDh + d), v);
        if (d == 0) {
          st_shared_cluster_u32(at + 4 * (kUnitHeads * kDh + h), __float_as_uint(m));
          st_shared_cluster_u32(at + 4 * (kUnitHeads * kDh + kUnitHeads + h), __float_as_uint(sum));
        }
      });
      cluster_sync();
      // (one CTA of the grid ends behind the prefix kernel, so that who waits for this kernel waits for that one too)
      if (C::kOwnOnly && blockIdx.x == gridDim.x - 1) pdl_wait();
      if (rank != 0) return;
      for (int i = tid; i < uh.count * (kDh / 4); i += kThreads) {
        const int h = i / (kDh / 4), d = (i % (kDh / 4)) * 4;
        float m = -INFINITY, sum = 0.0f;
        for (int r = 0; r < cs; ++r) m = fmaxf(m, all[r * kPart + kUnitHeads * kDh + h]);
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int r = 0; r < cs; ++r) {
          const float* const part = all + r * kPart;
          const float mr = part[kUnitHeads * kDh + h], f = mr == -INFINITY ? 0.0f : exp2_fast(mr - m);
          const float4 z = *reinterpret_cast<const float4*>(part + h * kDh + d);
          sum += part[kUnitHeads * kDh + kUnitHeads + h] * f;
          v.x += z.x * f;
          v.y += z.y * f;
          v.z += z.z * f;
          v.w += z.w * f;
        }
        write_out<C>(a, b, h0 + h, d, m, sum, v);
      }
      return;
    }
    if (tile == 0 && tile_end == tiles) {
      add_warps([&](int h, int d, float m, float sum, float4 v) { write_out<C>(a, b, h0 + h, d, m, sum, v); });
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

template <class C, int kNt>
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const typename C::Args a) {
  constexpr int kDh = C::kDh, kHeads = 8 * kNt, kBatch = 16, kJd = kDh / 32;  // parts; dimensions per lane
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
  const UnitHeads<C, kNt> uh(unit.y, group, parts);
  const int h0 = uh.h0;
  if (h >= uh.count) return;
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
  write_out<C>(a, unit.x, h0 + h, d, m, sum, v);
}

template <class C, int kNt>
constexpr size_t cluster_smem(int cs) {
  return (static_cast<size_t>(kWarps) * C::warp_floats(kNt) + static_cast<size_t>(cs) * C::kSplit * 8 * kNt * (C::kDh + 2)) * sizeof(float);
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
template <class C, int kNt>
SmemLimit& cluster_limit() {
  static SmemLimit limit;
  return limit;
}

// Clusters of cs CTAs that the GPU holds at once; 0 where it does not say.
template <class C, int kNt>
int clusters_at_once(int cs) {
  static DeviceNumber known[kMaxCluster + 1];
  ClusterLaunch l(1, cs, cluster_smem<C, kNt>(cs), nullptr);
  l.cfg.numAttrs = 1;
  return paged_clusters_at_once(known[cs], cluster_limit<C, kNt>(), reinterpret_cast<const void*>(paged_attention_kernel<C, kNt, true>),
                                cluster_smem<C, kNt>(kMaxCluster), l.cfg);
}

// A cluster of cs CTAs for each unit.
template <class C, int kNt>
cudaError_t launch_clusters(const typename C::Args& a, int units, int cs, cudaStream_t stream, unsigned int* launches) {
  cudaError_t e = cluster_limit<C, kNt>().allow(paged_attention_kernel<C, kNt, true>, cluster_smem<C, kNt>(kMaxCluster));
  if (e != cudaSuccess) return e;
  ClusterLaunch l(units, cs, cluster_smem<C, kNt>(cs), stream);
  if ((C::kOwnOnly || C::kHeadsOuter) && cs == 1) {  // (a CTA by itself finds a place sooner: 16 sequences of up to 96 x 40 heads 22.8 -> 21.8)
    l.attr[0] = l.attr[1];
    l.cfg.numAttrs = 1;
  }
  e = cudaLaunchKernelEx(&l.cfg, paged_attention_kernel<C, kNt, true>, a);
  if (e == cudaSuccess) ++*launches;
  return e;
}

template <class C, int kNt>
cudaError_t launch(const typename C::Args& a, cudaStream_t stream, unsigned int* launches) {
  constexpr size_t smem = static_cast<size_t>(kWarps) * C::warp_floats(kNt) * sizeof(float);
  // CTAs for every tile that the table has room for, at most a wave
  const int group = a.H / a.kv.Hkv;
  const long long units = static_cast<long long>(a.kv.Hkv / C::kSplit) * ((group + 8 * kNt - 1) / (8 * kNt)) * a.kv.seqs;
  constexpr int kTile = C::kTile;
  const long long room = std::max(1ll, ((static_cast<long long>(a.kv.table_cols) << a.kv.page_log2) + kTile - 1) / kTile);
  const int wave = std::min(kMaxGrid, num_sms() * C::ctas(kNt));
  // A cluster for each unit, if all have room at once (an eighth is left over: behind another kernel's last
  // CTAs 144 clusters of 3 took 23 us, of 2 17.7) and none of its CTAs has so many tiles more than equal ranges give
  // it, of sequences a third as long as the table, that the second kernel costs less. The table's width stands for the
  // lengths here, which the host does not know: 704 positions x 40 heads take 6.2 us in tables of up to 4096, 9.4 in
  // wider ones (8 heads 4.7, 8.7). us, with it and without: one sequence of 704 x 40 heads 6.2, 9.4, of 2048 x 8 6.5, 9.0, of 4096 x 8 11.0, 10.7, half as long as the table 4.1,
  // 7.9; 16 of up to 768 x 8 10.3, 13.7, 12 of up to 768 x 32 (12 tiles) 21.2, 19.6. A CTA for each of up to twice as many units of few tiles: 25 of 128 x 32
  // 14.2, 15.9, of 256 22.0, 23.5 (of five waves: 100 of 200 x 32 73, 66).
  // (Codes, whose tiles cost less: of up to three times as many units of up to eight tiles. 16 of up to 768 x 32 at 4 bits
  // 14.8, ranges 18.3, 30 of up to 300 x 32 at 8 16.4, 19.4, 64 of up to 900 x 8 at 4 18.5, 21.5.)
  const bool few = C::kHeadsOuter ? units <= 3 * wave && room <= 8 : units <= 2 * wave && room <= 2 * kMinTiles;
  if (C::kOwnOnly || units <= wave || few) {
    const bool spread = units * room <= num_sms();  // a tile each (256 x 32 heads 3.9, of two 4.8; 4 of 512 x 8 5.5, 4.9)
    int cs = static_cast<int>(std::min<long long>(kMaxCluster, spread ? room : (room + kMinTiles - 1) / kMinTiles));
    while (cs > 1 && units * 8 > clusters_at_once<C, kNt>(cs) * 7) --cs;
    // (Behind a prefix the table says nothing of the lengths.)
    if (C::kOwnOnly || (C::kHeadsOuter && few) || (room + cs - 1) / cs <= units * room / (3 * wave) + kJoinTiles)
      return launch_clusters<C, kNt>(a, static_cast<int>(units), cs, stream, launches);
  }
  if constexpr (C::kOwnOnly) {
    return cudaErrorInvalidValue;  // (not reached)
  } else {
    static SmemLimit limit;
    auto* kernel = paged_attention_kernel<C, kNt, false>;
    cudaError_t e = limit.allow(kernel, smem);
    if (e != cudaSuccess) return e;
    int grid = room >= wave || units >= wave ? wave : static_cast<int>(std::min<long long>(wave, units * room));
    if (C::kHeadsOuter && grid >= 8 * (units / a.kv.seqs)) grid -= grid % static_cast<int>(units / a.kv.seqs);
    e = launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads), smem, stream, a);
    if (e != cudaSuccess) return e;
    ++*launches;
    const unsigned heads = static_cast<unsigned>(C::kSplit > 1 ? C::kSplit * group : std::min(group, 8 * kNt));
    e = launch_pdl(join_kernel<C, kNt>, dim3(static_cast<unsigned>(grid), heads), dim3(32 * kJoinWarps), 0, stream,
                   a);
    if (e == cudaSuccess) ++*launches;
    return e;
  }
}

unsigned int read_and_clear_paged_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_paged_err, sizeof(v));
  cudaMemcpyToSymbol(g_paged_err, &z, sizeof(z));
  return v;
}

}  // namespace
}  // namespace p4q
