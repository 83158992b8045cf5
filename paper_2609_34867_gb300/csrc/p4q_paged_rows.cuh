// Attention over a paged cache of fp16 or bf16 keys and values: a warp's way through the
// tiles of a unit.
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
#pragma once

#include <type_traits>

#include "p4q_paged.cuh"
#include "p4q_paged_prefix.cuh"

namespace p4q {
namespace paged {

// p = 2^(score - reference + kShift), and a reference moves when a score exceeds it by
// 2^kMove. fp16: p up to 2^15, and small ones keep their bits (bf16 has fp32's range).
template <bool kBf16>
constexpr float kShift = kBf16 ? 0.0f : 11.0f;
template <bool kBf16>
constexpr float kMove = kBf16 ? 8.0f : 4.0f;

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

// Keys and values of 16 bits. kOwn: the positions from un.from on, which each sequence has
// of its own, behind a prefix.
template <bool kBf16Rows, int kDhRows, bool kSmallPage, bool kOwn = false>
struct Rows {
  typedef std::conditional_t<kOwn, PrefixArgs, PagedAttnArgs> Args;
  static constexpr bool kBf16 = kBf16Rows, kOwnOnly = kOwn, kHeadsOuter = false;
  static constexpr int kSplit = 1;
  static constexpr int kDh = kDhRows;
  static constexpr int kRep = 128 / kDh;  // blocks of 16 positions per warp and tile: 8 KB of keys and values
  static constexpr int kTile = 16 * kRep * kWarps;
  static constexpr int kKc = kDh / 32;    // 16-byte pieces of a key row per lane
  static constexpr int kVc = kDh / 64;    // of a value row
  static constexpr float kLift = kShift<kBf16>;
  static __host__ __device__ constexpr int warp_floats(int nt) { return 8 * nt * kDh; }  // (for its part of O)
  static __host__ __device__ constexpr int ctas(int nt) { return nt == 1 ? 3 : 2; }
  static __device__ __forceinline__ bool bf16(const Args&) { return kBf16; }
  typedef std::conditional_t<kOwn, PrefixOf, NoPrefix> Behind;
  static __device__ __forceinline__ int first_dim(int hh, int g) { return 64 * hh + 8 * g; }

  // Goes through tiles tile .. tile_end - 1 of the unit. sq: the warp's place for the query operand.
  template <int kNt>
  static __device__ __forceinline__ void attend(const Args& a, const Unit& un, int tile, int tile_end,
                                                uint4 (&sq)[kNt][kKc][32], float*, Part<kNt, kVc>& acc) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const float c2 = a.scale * 1.4426950408889634f;
    const PagedCache& c = a.kv;
    const int len = un.len, heads = un.heads;
    if (kOwn && un.from >= len) return;  // (nothing behind the prefix)
    const uint16_t* kh = c.k + un.hk * c.head_stride + t * 8;
    const uint16_t* vh = c.v + un.hk * c.head_stride + g * 8;
    const int slots = (1 << c.page_log2) - 1;

    // Element offset of position j in the cache (without the head), -1 if it is not to be read.
    auto offset = [&](int j) -> long long {
      if (j >= len || (kOwn && kSmallPage && j < un.from)) return -1;
      const int page = un.table[j >> c.page_log2];
      if (static_cast<unsigned int>(page) >= static_cast<unsigned int>(c.pages)) {
        atomicOr(&g_paged_err, kErrIndex);
        return -1;
      }
      return page * c.page_stride + (j & slots) * c.token_stride;
    };

    auto& o = acc.o;
    auto& ref = acc.ref;
    auto& l = acc.l;
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
        const int j = un.base + tl * kTile + (warp * kRep + r) * 16;
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
        const int j = un.base + tl * kTile + (warp * kRep + r) * 16;
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
          const int from = kOwn ? un.from : 0;
          live |= (j + g < len && (!kOwn || j + g >= from) ? 1u << (2 * r) : 0u) |
                  (j + g + 8 < len && (!kOwn || j + g + 8 >= from) ? 2u << (2 * r) : 0u);
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

    if (tile < tile_end) look(tile);
    // Q: head g of each 8, dimensions 32 i + 8 t .. (on its way beside the page numbers)
    uint4 q[kNt][kKc];
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int i = 0; i < kKc; ++i) {
        const int h = 8 * n + g;
        q[n][i] = make_uint4(0u, 0u, 0u, 0u);
        if (h < heads) q[n][i] = *reinterpret_cast<const uint4*>(a.q + un.b * a.ldq + static_cast<long long>(un.h0 + h) * kDh + 32 * i + 8 * t);
      }
    if (tile < tile_end) {
      load_k(tile);
      load_v(tile);
      look(tile + 1);
    }
    __syncwarp();
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int i = 0; i < kKc; ++i) sq[n][i][lane] = q[n][i];
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
            const uint4 f = reload16(&sq[n][i][lane]);
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
  }
};

}  // namespace paged
}  // namespace p4q
