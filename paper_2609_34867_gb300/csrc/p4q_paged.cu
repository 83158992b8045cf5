// Attention of one new token per sequence over a paged key/value cache:
//   o_h = sum_{j < len} p_j v_j,  p = softmax_j(scale q_h . k_j).
//
// Work: a unit is one key/value head of one sequence with up to 8 NT of the
// query heads that share it (a group of more heads makes several units), cut
// into tiles of positions. All units' tiles in one row, unit after unit, are
// dealt to the CTAs in equal consecutive ranges, so a CTA's work does not
// depend on how unequal the sequences are; a unit that several CTAs share is
// joined by the one that finishes last.
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
// 2^8 (p stays below 2^15), so that most tiles need no exchange between lanes.
// p goes into the product as the sum of two 16-bit values (rounded, remainder):
// rounded once it would add as much error as the output's own rounding does.
// The new keys' loads are issued as soon as the old ones are in the first
// product, and the values' behind the second.
#include <cuda_runtime.h>

#include <algorithm>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {

__device__ unsigned int g_paged_err;

namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxGrid = 512;    // CTAs of a launch at most (partial results of the workspace)
constexpr int kMinTiles = 2;     // tiles per CTA at least, unless there are fewer
constexpr float kShift = 7.0f;   // p = 2^(score - reference + 7): small p keep their bits in fp16
constexpr float kMove = 8.0f;    // a reference moves when a score exceeds it by 2^8

// Workspace: a counter per CTA (zero between calls), then two partial results
// per CTA: 16 maxima, 16 sums, 16 x 128 values.
constexpr int kPartFloats = 32 + 16 * 128;
constexpr size_t kWsBytes = kMaxGrid * sizeof(int) + static_cast<size_t>(kMaxGrid) * 2 * kPartFloats * sizeof(float);

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

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint4 load16(const uint16_t* p, bool valid) {
  return valid ? ldg_stream16(p) : make_uint4(0u, 0u, 0u, 0u);
}

struct Plan {  // what a CTA computes from the lengths
  long long total;   // tiles of all units
  long long first;   // this CTA's tiles: first .. last - 1
  long long last;
  int grid;          // CTAs that have a range
  int b, u, tile;    // where `first` lies
};

template <bool kBf16, int kDh, int kNt, bool kSmallPage>
__global__ void __launch_bounds__(kThreads, kNt == 1 ? 2 : 1) paged_attention_kernel(const PagedAttnArgs a) {
  constexpr int kHeads = 8 * kNt;
  constexpr int kRep = 128 / kDh;          // blocks of 16 positions per warp and tile: 8 KB of keys and values
  constexpr int kTile = 16 * kRep * kWarps;
  constexpr int kKc = kDh / 32;            // 16-byte pieces of a key row per lane
  constexpr int kVc = kDh / 64;            // of a value row
  extern __shared__ __align__(16) float so[];  // [kWarps][kHeads][kDh]
  __shared__ float sm[kWarps][kHeads], sl[kWarps][kHeads];
  __shared__ long long scan[kWarps + 1];
  __shared__ Plan plan;
  __shared__ int joined;

  const PagedCache& c = a.kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int group = a.H / c.Hkv, parts = (group + kHeads - 1) / kHeads, units = c.Hkv * parts;
  const long long room = static_cast<long long>(c.table_cols) << c.page_log2;
  const float c2 = a.scale * 1.4426950408889634f;
  int* counters = static_cast<int*>(a.ws);
  float* partial = reinterpret_cast<float*>(counters + kMaxGrid);

  pdl_wait();
  pdl_launch_dependents();

  auto length = [&](int b) -> int {
    const int n = a.lens[b];
    return n < 0 ? 0 : n > room ? static_cast<int>(room) : n;
  };
  auto tiles_of = [&](int n) { return n <= kTile ? 1 : (n + kTile - 1) / kTile; };

  // The tiles before this thread's sequences, their sum, and from these the
  // CTA's range and where it begins.
  {
    const int per = (c.seqs + kThreads - 1) / kThreads, b0 = min(c.seqs, tid * per), b1 = min(c.seqs, b0 + per);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) {
      if (a.lens[b] > room && blockIdx.x == 0) atomicOr(&g_paged_err, kErrIndex);
      mine += tiles_of(length(b));
    }
    long long upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto += v;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) upto += scan[w];
      all += scan[w];
    }
    const long long total = all * units;
    const int grid = static_cast<int>(max(1ll, min(static_cast<long long>(gridDim.x), total / kMinTiles)));
    const int cta = static_cast<int>(blockIdx.x);
    if (cta >= grid) return;  // (the whole CTA)
    const long long first = total * cta / grid, last = total * (cta + 1) / grid;
    if (first >= (upto - mine) * units && first < upto * units) {
      long long at = (upto - mine) * units;
      for (int b = b0; b < b1; ++b) {
        const int n = tiles_of(length(b));
        if (first < at + static_cast<long long>(n) * units) {
          plan.b = b;
          plan.u = static_cast<int>((first - at) / n);
          plan.tile = static_cast<int>((first - at) % n);
          break;
        }
        at += static_cast<long long>(n) * units;
      }
      plan.total = total;
      plan.first = first;
      plan.last = last;
      plan.grid = grid;
    }
    __syncthreads();
  }

  long long x = plan.first;
  int b = plan.b, u = plan.u, tile = plan.tile;
  while (x < plan.last) {
    const int len = length(b), tiles = tiles_of(len);
    const int tile_end = static_cast<int>(min(static_cast<long long>(tiles), tile + (plan.last - x)));
    const int hk = u / parts, h0 = hk * group + (u % parts) * kHeads;
    const int heads = min(kHeads, hk * group + group - h0);
    const int32_t* table = c.table + static_cast<long long>(b) * c.table_ld;
    const uint16_t* kh = c.k + hk * c.head_stride + t * 8;
    const uint16_t* vh = c.v + hk * c.head_stride + g * 8;
    const int slots = (1 << c.page_log2) - 1;

    // Element offset of position j (in the cache, without the head), -1 if it is not to be read.
    auto offset = [&](int j) -> long long {
      if (j >= len) return -1;
      const int page = table[j >> c.page_log2];
      if (static_cast<unsigned int>(page) >= static_cast<unsigned int>(c.pages)) {
        atomicOr(&g_paged_err, kErrIndex);
        return -1;
      }
      return page * c.page_stride + (j & slots) * c.token_stride;
    };

    uint32_t qf[kNt][kKc][4];  // Q: head g of each 8, dimensions 32 i + 8 t ..
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int i = 0; i < kKc; ++i) {
        const int h = 8 * n + g;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (h < heads) v = *reinterpret_cast<const uint4*>(a.q + b * a.ldq + static_cast<long long>(h0 + h) * kDh + 32 * i + 8 * t);
        qf[n][i][0] = v.x;
        qf[n][i][1] = v.y;
        qf[n][i][2] = v.z;
        qf[n][i][3] = v.w;
      }

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
    // offset is looked up a tile ahead of its loads. With smaller pages each
    // row's is.
    constexpr int kLook = kSmallPage ? 6 : 1;
    long long off[kRep][kLook];
    uint32_t live = 0;  // bits 2 rep, 2 rep + 1: the keys of rows g, g + 8 of the loaded blocks count
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
    auto load_k = [&](int tl) {
      live = 0;
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        const int j = tl * kTile + (warp * kRep + r) * 16;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const long long at = kSmallPage ? off[r][e] : off[r][0] + (g + 8 * e) * c.token_stride;
          const bool valid = kSmallPage ? off[r][e] >= 0 : (off[r][0] >= 0 && j + g + 8 * e < len);
          live |= valid ? 1u << (2 * r + e) : 0u;
#pragma unroll
          for (int i = 0; i < kKc; ++i) kr[r][i][e] = load16(kh + at + 32 * i, valid);
        }
      }
    };
    auto load_v = [&](int tl) {
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        const int j = tl * kTile + (warp * kRep + r) * 16;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 2 * t + (e & 1) + 4 * (e & 2);
          const long long at = kSmallPage ? off[r][2 + e] : off[r][0] + row * c.token_stride;
          const bool valid = kSmallPage ? off[r][2 + e] >= 0 : (off[r][0] >= 0 && j + row < len);
#pragma unroll
          for (int hh = 0; hh < kVc; ++hh) vr[r][hh][e] = load16(vh + at + 64 * hh, valid);
        }
      }
    };

    look(tile);
    load_k(tile);
    load_v(tile);
    look(tile + 1);
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
            mma16816<kBf16>(s[r][n], kr[r][i][0].x, kr[r][i][1].x, kr[r][i][0].y, kr[r][i][1].y, qf[n][i][0], qf[n][i][1]);
            mma16816<kBf16>(s[r][n], kr[r][i][0].z, kr[r][i][1].z, kr[r][i][0].w, kr[r][i][1].w, qf[n][i][2], qf[n][i][3]);
          }
        }
      const uint32_t counts = live;
      if (more) load_k(tl + 1);
      // scores in powers of two; positions that do not count have none
      bool move = false;
#pragma unroll
      for (int r = 0; r < kRep; ++r)
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = (counts >> (2 * r + (e >> 1)) & 1u) ? s[r][n][e] * c2 : -INFINITY;
            s[r][n][e] = y;
            move = move || y > ref[n][e & 1] + kMove;
          }
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
        for (int e = 0; e < 2; ++e) from[n][e] = ref[n][e] == -INFINITY ? 0.0f : ref[n][e] - kShift;
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        uint32_t bh[kNt][2], bl[kNt][2];
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {  // rows g, g + 8
            const float p0 = exp2_fast(s[r][n][2 * e] - from[n][0]), p1 = exp2_fast(s[r][n][2 * e + 1] - from[n][1]);
            l[n][0] += p0;
            l[n][1] += p1;
            const uint32_t hi = pack2<kBf16>(p0, p1);
            const float2 back = unpack2<kBf16>(hi);
            bh[n][e] = transpose8x8(hi);
            bl[n][e] = transpose8x8(pack2<kBf16>(p0 - back.x, p1 - back.y));
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
            for (int n = 0; n < kNt; ++n) {
              mma16816<kBf16>(o[n][hh][j], a0, a1, a2, a3, bh[n][0], bh[n][1]);
              mma16816<kBf16>(o[n][hh][j], a0, a1, a2, a3, bl[n][0], bl[n][1]);
            }
          }
        }
      }
      if (more) {
        load_v(tl + 1);
        look(tl + 2);
      }
    }

    // The CTA's warps joined: each scales its part to the largest reference.
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, l[n][e], d);
        if (g == 0) {
          sm[warp][8 * n + 2 * t + e] = ref[n][e];
          sl[warp][8 * n + 2 * t + e] = l[n][e];
        }
      }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int h = 8 * n + 2 * t + e;
        float m = sm[0][h];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm[w][h]);
        const float f = ref[n][e] == -INFINITY ? 0.0f : exp2_fast(ref[n][e] - m);
        if (h < heads) {
#pragma unroll
          for (int hh = 0; hh < kVc; ++hh) {
            float* d = so + (warp * kHeads + h) * kDh + 64 * hh + 8 * g;
#pragma unroll
            for (int j = 0; j < 4; j += 2)
              *reinterpret_cast<float4*>(d + 2 * j) = make_float4(o[n][hh][j][e] * f, o[n][hh][j][e + 2] * f,
                                                                  o[n][hh][j + 1][e] * f, o[n][hh][j + 1][e + 2] * f);
          }
        }
      }
    __syncthreads();

    // (head, four dimensions) per thread and step: maximum, sum and values
    auto write = [&](int h, int d, float m, float sum, float4 v) {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      uint2 w;
      w.x = pack2<kBf16>(v.x * inv, v.y * inv);
      w.y = pack2<kBf16>(v.z * inv, v.w * inv);
      *reinterpret_cast<uint2*>(a.o + b * a.ldo + static_cast<long long>(h0 + h) * kDh + d) = w;
      if (d == 0 && a.lse)
        a.lse[static_cast<long long>(b) * a.H + h0 + h] =
            sum == 0.0f ? -INFINITY : (m - kShift) * 0.6931471805599453f + logf(sum);
    };
    const bool whole = tile == 0 && tile_end == tiles;
    const int cta = static_cast<int>(blockIdx.x);
    float* part = partial + static_cast<size_t>(2 * cta + (tile == 0 ? 1 : 0)) * kPartFloats;
    for (int i = tid; i < heads * (kDh / 4); i += kThreads) {
      const int h = i / (kDh / 4), d = (i % (kDh / 4)) * 4;
      float m = sm[0][h], sum = 0.0f;
#pragma unroll
      for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm[w][h]);
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = sm[w][h] == -INFINITY ? 0.0f : exp2_fast(sm[w][h] - m);
        sum += sl[w][h] * f;
        const float4 z = *reinterpret_cast<const float4*>(so + (w * kHeads + h) * kDh + d);
        v.x += z.x;
        v.y += z.y;
        v.z += z.z;
        v.w += z.w;
      }
      if (whole) {
        write(h, d, m, sum, v);
      } else {
        if (d == 0) {
          part[h] = m;
          part[16 + h] = sum;
        }
        *reinterpret_cast<float4*>(part + 32 + h * kDh + d) = v;
      }
    }
    if (!whole) {
      // The unit's CTAs: c0 (whose part is the second of its two) .. c1.
      const long long x0 = x - tile;
      const int c0 = static_cast<int>(((x0 + 1) * plan.grid - 1) / plan.total);
      const int c1 = static_cast<int>(((x0 + tiles) * plan.grid - 1) / plan.total);
      __threadfence();
      __syncthreads();
      if (tid == 0) joined = atomicAdd(counters + c0, 1) == c1 - c0;
      __syncthreads();
      if (joined) {
        __threadfence();
        for (int i = tid; i < heads * (kDh / 4); i += kThreads) {
          const int h = i / (kDh / 4), d = (i % (kDh / 4)) * 4;
          float m = -INFINITY, sum = 0.0f;
          float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int k = c0; k <= c1; ++k) m = fmaxf(m, __ldcg(partial + static_cast<size_t>(2 * k + (k == c0)) * kPartFloats + h));
          for (int k = c0; k <= c1; ++k) {
            const float* p = partial + static_cast<size_t>(2 * k + (k == c0)) * kPartFloats;
            const float mk = __ldcg(p + h), f = mk == -INFINITY ? 0.0f : exp2_fast(mk - m);
            const float4 z = __ldcg(reinterpret_cast<const float4*>(p + 32 + h * kDh + d));
            sum += __ldcg(p + 16 + h) * f;
            v.x += z.x * f;
            v.y += z.y * f;
            v.z += z.z * f;
            v.w += z.w * f;
          }
          write(h, d, m, sum, v);
        }
        if (tid == 0) counters[c0] = 0;  // ready for the next call
      }
    }
    __syncthreads();  // the shared results have been read

    x += tile_end - tile;
    tile = 0;
    if (++u == units) {
      u = 0;
      ++b;
    }
  }
}

template <bool kBf16, int kDh, int kNt, bool kSmallPage>
cudaError_t launch(const PagedAttnArgs& a, cudaStream_t stream) {
  constexpr size_t smem = static_cast<size_t>(kWarps) * 8 * kNt * kDh * sizeof(float);
  static SmemLimit limit;
  auto* kernel = paged_attention_kernel<kBf16, kDh, kNt, kSmallPage>;
  if (smem > 32 * 1024) {
    const cudaError_t e = limit.allow(kernel, smem);
    if (e != cudaSuccess) return e;
  }
  // CTAs for every tile that the table has room for, at most a wave
  const int group = a.H / a.kv.Hkv;
  const long long units = static_cast<long long>(a.kv.Hkv) * ((group + 8 * kNt - 1) / (8 * kNt)) * a.kv.seqs;
  constexpr int kTile = 16 * (128 / kDh) * kWarps;
  const long long room = std::max(1ll, ((static_cast<long long>(a.kv.table_cols) << a.kv.page_log2) + kTile - 1) / kTile);
  const int wave = std::min(kMaxGrid, num_sms() * (kNt == 1 ? 2 : 1));
  const int grid = room >= wave || units >= wave ? wave : static_cast<int>(std::min<long long>(wave, units * room));
  return launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads), smem, stream, a);
}

template <bool kBf16, int kDh>
cudaError_t launch_for(const PagedAttnArgs& a, cudaStream_t stream) {
  const bool wide = a.H / a.kv.Hkv > 8, small = a.kv.page_log2 < 4;
  if (wide) return small ? launch<kBf16, kDh, 2, true>(a, stream) : launch<kBf16, kDh, 2, false>(a, stream);
  return small ? launch<kBf16, kDh, 1, true>(a, stream) : launch<kBf16, kDh, 1, false>(a, stream);
}

}  // namespace

size_t paged_attention_workspace_bytes() { return kWsBytes; }

cudaError_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t stream) {
  if (a.kv.bf16) return a.kv.dh == 64 ? launch_for<true, 64>(a, stream) : launch_for<true, 128>(a, stream);
  return a.kv.dh == 64 ? launch_for<false, 64>(a, stream) : launch_for<false, 128>(a, stream);
}

unsigned int paged_read_and_clear_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_paged_err, sizeof(v));
  cudaMemcpyToSymbol(g_paged_err, &z, sizeof(z));
  return v;
}

}  // namespace p4q
