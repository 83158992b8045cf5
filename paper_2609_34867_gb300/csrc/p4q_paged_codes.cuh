// Attention over a paged cache of 8- or 4-bit codes with one scale per position and head: a
// warp's way through the tiles of a unit.
//   x_j = (scale log2 e) sk_j (q . c_j),  p_j = 2^(x_j - ref),  o = sum_j (p_j sv_j) c'_j / sum_j p_j
// with codes c_j, c'_j and scales sk_j, sv_j of key and value: the codes enter the products as
// they are (whole numbers, exact in fp16) and the scales are factors of the positions' scores
// and weights, four multiplications per 16 positions and lane.
//
// A warp takes 16 positions at a time as operands of m16n8k16 products, positions the rows of
// S^T = K Q^T and the inner axis of O^T = V^T P^T. Keys, values and scales of its next one or two
// tiles are on their way into a ring of its own in shared memory meanwhile, by asynchronous
// copies (straight into registers, as 16-bit rows go, half a tile ahead: with codes a tile's bytes
// are too few to cover the latency, 24 sequences of up to 2048 x 40 heads at 8 bits 64 us, 54 this way).
// Codes become fp16 in registers: a byte or nibble is the low mantissa bits of
// 1024 (nibbles in the high half of a byte: of 1024 / 16 = 64, undone by the multiplication that
// takes the offset away), one logical operation and one packed addition for two codes. Which
// dimensions an MMA's k-th ones are is free as long as q has the same order, so the nibbles
// {0, 4}, {1, 5}, {2, 6}, {3, 7} of a word are pairs as they lie.
//
// q enters the product in fp16: with 8 bits q of fp16 as it is, else times the power of two that
// brings its head's largest finite value below 2^15: exact where |q| is not below 2^-25 of that one, and
// off by less than 2^-35 of it elsewhere. The weights p sv enter theirs as two fp16 values (22 bits)
// times a power of two per head that moves like the softmax's reference and with it, so scales of any
// size count against the largest p sv seen, each at its weight now, and not against fp16's range.
//
// What bounds it. 8 bits: HBM, 24 ragged sequences of up to 2048 x 40 heads 52 - 55 us, 0.72 - 0.77 of a copy's
// rate (loads of single heads' rows by two stages; 16-bit rows, twice as long, reach 0.92). 4 bits: instructions and their latencies at twelve
// warps per SM, about 300 per block of 16 positions of 128 (537 in the first version, with codes converted to
// whole numbers one by one), 158 cycles of an SM against 93 of HBM: 128 sequences of up to 8190 x 8 heads 79 us,
// 0.55 (77.5 with scores that were not rounded before the reference is taken off and a factor of the weights that did
// not follow it). Tried at 77: tiles of one block and four CTAs of 126 registers 87, of four blocks 84 - 108; values'
// nibbles too as what fp16 reads in them, their 8s taken back by products with the weights 80, by sums per tile (23
// instructions fewer) 77, so not worth their rounding.
#pragma once

#include "p4q_paged.cuh"

namespace p4q {
namespace paged {

// Constants that the compiler is to keep in registers: an instruction has room for one of its own, and
// it would rather use two of these (64 more per block of 16 positions at 4 bits).
struct Magic {
  uint32_t lo, hi, key_lo, key_hi, bytes;
  __device__ __forceinline__ Magic() {
    asm volatile("mov.b32 %0, 0x64086408;" : "=r"(lo));
    asm volatile("mov.b32 %0, 0x64806480;" : "=r"(hi));
    asm volatile("mov.b32 %0, 0x00080008;" : "=r"(key_lo));
    asm volatile("mov.b32 %0, 0x00800080;" : "=r"(key_hi));
    asm volatile("mov.b32 %0, 0x64646464;" : "=r"(bytes));
  }
};

// Two codes as fp16 pairs. Bytes 2 half, 2 half + 1 of a word whose sign bits are flipped.
template <int kHalf>
__device__ __forceinline__ uint32_t codes8(uint32_t flipped, const Magic& k) {
  const uint32_t v = __byte_perm(flipped, k.bytes, kHalf ? 0x4342 : 0x4140);  // 1024 + 128 + c
  const uint32_t bias = 0x64806480u;
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&bias));
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Nibbles kOdd of both 16-bit halves (0: bits 0 - 3, 1: bits 4 - 7).
template <int kOdd>
__device__ __forceinline__ uint32_t codes4(uint32_t w, const Magic& k) {
  __half2 h;
  uint32_t v;
  if (kOdd) {
    const uint32_t f = 0x2C002C00u, bias = 0xD480D480u;
    asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0x6A;" : "=r"(v) : "r"(w), "r"(k.hi));  // 1024 + 16 (8 + c); 1/16; -72
    h = __hfma2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&f),
                *reinterpret_cast<const __half2*>(&bias));
  } else {
    const uint32_t bias = 0x64086408u;
    asm("lop3.b32 %0, %1, 0x000F000F, %2, 0x6A;" : "=r"(v) : "r"(w), "r"(k.lo));  // 1024 + 8 + c
    h = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&bias));
  }
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Asynchronous copies to shared memory. kHalfLines: fetched 64 bytes at a time, where the other half of a
// 128-byte line is of no use soon: whole lines moved 1.65 times the bytes from HBM where a position's
// codes are 64 and other heads' lie between (64 x 4096 x 8 heads at 4 bits 95 us instead of 71).
template <bool kHalfLines>
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src) {
  if (kHalfLines)
    asm volatile("cp.async.cg.shared.global.L2::64B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
template <bool kHalfLines>
__device__ __forceinline__ void copy4(uint32_t dst, const float* src) {
  if (kHalfLines)
    asm volatile("cp.async.ca.shared.global.L2::64B [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// The same nibbles of keys as what fp16 reads in them: (8 + c) 2^-24, 16 times that of the odd ones. Exact in
// the product; q takes the factor 16 and the accumulator begins with what the 8 adds.
template <int kOdd>
__device__ __forceinline__ uint32_t key_codes4(uint32_t w, const Magic& k) {
  uint32_t v;
  if (kOdd)
    asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0x6A;" : "=r"(v) : "r"(w), "r"(k.key_hi));
  else
    asm("lop3.b32 %0, %1, 0x000F000F, %2, 0x6A;" : "=r"(v) : "r"(w), "r"(k.key_lo));
  return v;
}

template <int kWords>
__device__ __forceinline__ void read_words(uint32_t* w, uint32_t at) {
  if constexpr (kWords == 4)
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
  else if constexpr (kWords == 2)
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  else
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}

// kPair: at most four heads to a key/value head's unit. Columns 4 - 7 of the products, which would be
// empty, then repeat heads 0 - 3 and take the second fp16 value of their weights, so one product
// of O^T does for both.
// kSplit: the warps of a CTA take that many neighbouring key/value heads turn by turn, whose codes of a
// position share a line of HBM.
template <int kBits, int kDhRows, bool kSmallPage, bool kPair, int kSplitHeads>
struct Codes {
  typedef QuantAttnArgs Args;
  static constexpr bool kOwnOnly = false, kHeadsOuter = true;
  static constexpr int kDh = kDhRows;
  static constexpr int kRep = kDh * kBits == 1024 ? 1 : kDh * kBits == 256 && !kSmallPage ? 4 : 2;  // blocks of 16 positions per warp and tile
  static constexpr int kSplit = kSplitHeads;
  static constexpr int kTile = 16 * kRep * kWarps / kSplit;
  static constexpr int kKc = kDh / 32;             // pieces of q per lane, 8 dimensions each
  static constexpr int kVc = kDh / 64;
  static constexpr int kKw = kDh * kBits / 128;    // words of a key row per lane
  static constexpr int kVw = kDh * kBits / 256;    // of a value row
  static constexpr int kRow = kDh * kBits / 8;     // bytes of a row
  static constexpr int kChunks = kRow / 16;        // copies of 16 bytes for it
  static constexpr int kAtOnce = 32 / kChunks;     // rows that a warp copies at once
  static constexpr int kBlock = 32 * kRow + 128;   // bytes of 16 positions: keys, values, scales
  static constexpr int kStages = kRow == 128 ? 2 : 3;
  static constexpr bool kHalf = kRow * kSplit < 128;
  // Floats of a warp's ring of stages; its part of O takes their place in the end.
  static __host__ __device__ constexpr int warp_floats(int nt) {
    return kStages * kRep * kBlock / 4 > 8 * nt * kDh ? kStages * kRep * kBlock / 4 : 8 * nt * kDh;
  }
  // Where chunk ch of row r lies in a row's place: eight lanes that read rows and chunks as the
  // products want them find them in eight banks' groups.
  static __device__ __forceinline__ int place(int r, int ch) {
    return r * kRow + ((kChunks == 8 ? ch ^ (r & 7) : kChunks == 4 ? ch ^ (r >> 1 & 3) : ch) << 4);
  }
  static constexpr float kLift = 0.0f;
  static constexpr float kMove = 8.0f;
  static constexpr int kSecond = kPair ? 1 : 2;    // products per operand of O^T
  static __host__ __device__ constexpr int ctas(int nt) { return nt == 2 ? 2 : kDh * kBits == 1024 && !kSmallPage ? 4 : 3; }
  static __device__ __forceinline__ bool bf16(const Args& a) { return a.bf16; }
  typedef NoPrefix Behind;
  static __device__ __forceinline__ int first_dim(int hh, int g) { return (kDh / 8) * g + 8 * hh; }
  // The dimensions of q's piece p that lane t's keys have.
  static __device__ __forceinline__ int q_dim(int p, int t) { return (kDh / 4) * t + 8 * p; }

  template <int kNt>
  static __device__ __forceinline__ void attend(const Args& a, const Unit& un, int tile, int tile_end,
                                                uint4 (&sq)[kNt][kKc][32], float* ring, Part<kNt, kVc>& acc) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const PagedCodes& c = a.kv;
    const Magic magic;
    const int len = un.len, heads = un.heads;
    const int slots = (1 << c.page_log2) - 1;
    // The lane copies chunk `chunk` of rows `sub`, sub + kAtOnce, .. of keys and values, and of the scales of
    // row lane % 16 the key's (lanes 0 - 15) or the value's. With small pages the rows are added at the copy.
    const int chunk = lane % kChunks, sub = lane / kChunks;
    const long long ts = c.token_stride, ss = c.scale_token_stride;
    const uint8_t* const kh = c.k + un.hk * c.head_stride + (kSmallPage ? 0 : sub * ts) + 16 * chunk;
    const uint8_t* const vh = c.v + un.hk * c.head_stride + (kSmallPage ? 0 : sub * ts) + 16 * chunk;
    const float* const sh = (lane < 16 ? c.k_scale : c.v_scale) + un.hk * c.scale_head_stride + (kSmallPage ? 0 : (lane & 15) * ss);
    const uint32_t slots_at = smem_u32(ring);
    const uint32_t scale_to = 32 * kRow + 4 * (16 * (lane >> 4) + 2 * (lane & 7) + (lane >> 3 & 1));  // rows g, g + 8 side by side
    auto block_at = [&](int tl, int r) { return tl * kTile + (warp / kSplit * kRep + r) * 16; };

    // The page of position j, -1 if it is not to be read.
    auto page_of = [&](int j) -> int {
      if (j >= len) return -1;
      const int page = un.table[j >> c.page_log2];
      if (static_cast<unsigned int>(page) >= static_cast<unsigned int>(c.pages)) {
        atomicOr(&g_paged_err, kErrIndex);
        return -1;
      }
      return page;
    };

    auto& o = acc.o;
    auto& l = acc.l;
    // Pages of 16 and more: a block of 16 positions lies in one, and each lane has the place of one of
    // the warp's next 32 blocks (and the page of one of the 32 after them), found once for all lanes.
    // Smaller pages: of one of the next 32 positions.
    static_assert(!kSmallPage || kRep <= 2, "at most 32 positions of a warp in a tile");
    constexpr int kStrip = kSmallPage ? 1 : 32 / kRep;  // tiles
    int strip = tile, page_ahead = -1;
    long long code_at = 0, scale_at = 0;
    uint32_t found = 0;  // the strip's blocks (positions) that are to be read
    auto mine_at = [&](int tl) { return kSmallPage ? block_at(tl, 0) + lane : block_at(tl + lane / kRep, lane % kRep); };
    auto look = [&](int tl) {
      page_ahead = tl + (kSmallPage ? 0 : lane / kRep) < tile_end && (!kSmallPage || lane < 16 * kRep) ? page_of(mine_at(tl)) : -1;
    };
    auto enter_strip = [&](int tl) {
      strip = tl;
      found = __ballot_sync(0xFFFFFFFFu, page_ahead >= 0);
      const long long slot = mine_at(tl) & slots;
      code_at = page_ahead * c.page_stride + slot * ts;
      scale_at = page_ahead * c.scale_page_stride + slot * ss;
      look(tl + kStrip);
    };
    // Copies tile tl into its stage, and says which of the blocks there are (small pages: positions).
    auto copy = [&](int tl, int stage) -> uint32_t {
      if (tl - strip == kStrip) enter_strip(tl);
      const int first = (tl - strip) * kRep;
      const uint32_t there = kSmallPage ? found : found >> first & ((1u << kRep) - 1u);
      const uint32_t to = slots_at + stage * (kRep * kBlock);
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        if constexpr (kSmallPage) {
#pragma unroll
          for (int i = 0; i < 16 / kAtOnce; ++i) {
            const int row = i * kAtOnce + sub;
            const long long at = __shfl_sync(0xFFFFFFFFu, code_at, 16 * r + row);
            if (there >> (16 * r + row) & 1u) {
              copy16<kHalf>(to + r * kBlock + place(row, chunk), kh + at);
              copy16<kHalf>(to + r * kBlock + 16 * kRow + place(row, chunk), vh + at);
            }
          }
          const long long at = __shfl_sync(0xFFFFFFFFu, scale_at, 16 * r + (lane & 15));
          if (there >> (16 * r + (lane & 15)) & 1u) copy4<kHalf>(to + r * kBlock + scale_to, sh + at);
        } else {
          const long long at = __shfl_sync(0xFFFFFFFFu, code_at, first + r), sat = __shfl_sync(0xFFFFFFFFu, scale_at, first + r);
          if (there >> r & 1u) {  // (rows past the length are read too: they are the page's)
#pragma unroll
            for (int i = 0; i < 16 / kAtOnce; ++i) {
              const uint32_t d = to + r * kBlock + place(i * kAtOnce + sub, chunk);
              copy16<kHalf>(d, kh + at + i * kAtOnce * ts);
              copy16<kHalf>(d + 16 * kRow, vh + at + i * kAtOnce * ts);
            }
            copy4<kHalf>(to + r * kBlock + scale_to, sh + sat);
          }
        }
      }
      return there;
    };
    // Which rows of a tile count, where not all of them do (all: bits 2 r, 2 r + 1 for rows g, g + 8 of block r).
    constexpr uint32_t kAll = (1u << (2 * kRep)) - 1u;
    auto counting = [&](int tl, uint32_t there) -> uint32_t {
      constexpr uint32_t kThere = kSmallPage ? (kRep == 2 ? 0xFFFFFFFFu : 0xFFFFu) : (1u << kRep) - 1u;
      if (there == kThere && block_at(tl, kRep) <= len) return kAll;
      uint32_t live = 0;
#pragma unroll
      for (int r = 0; r < kRep; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = g + 8 * e;
          if (kSmallPage ? there >> (16 * r + row) & 1u : (there >> r & 1u) && block_at(tl, r) + row < len) live |= 1u << (2 * r + e);
        }
      return live;
    };
    uint32_t there_of[kStages];  // of the stages' tiles, the oldest first

    if (tile < tile_end) look(tile);
    uint4 raw[kNt][kKc];  // q: head g of each 8 (on its way beside the page numbers)
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int p = 0; p < kKc; ++p) {
        const int h = kPair ? g & 3 : 8 * n + g;
        raw[n][p] = make_uint4(0u, 0u, 0u, 0u);
        if (h < heads)
          raw[n][p] = *reinterpret_cast<const uint4*>(a.q + un.b * a.ldq + static_cast<long long>(un.h0 + h) * kDh + q_dim(p, t));
      }
    if (tile < tile_end) {
      enter_strip(tile);
#pragma unroll
      for (int i = 0; i < kStages - 1; ++i) {
        there_of[i] = tile + i < tile_end ? copy(tile + i, i) : 0u;
        cp_async_commit();
      }
    }
    // q as fp16 (times the sign of the scale, or 0), and the factor fq >= 0 that makes scores in powers of
    // two of its products with a position's codes and scale (heads 2 t, 2 t + 1)
    const float c2 = fabsf(a.scale * 1.4426950408889634f), sign = a.scale > 0.0f ? 1.0f : a.scale < 0.0f ? -1.0f : 0.0f;
    float fq[kNt][2], begin[kNt][2] = {};  // and what the products' sums begin with
    __syncwarp();
#pragma unroll
    for (int n = 0; n < kNt; ++n) {
      uint4 (&q)[kKc] = raw[n];
      float f = c2 == 0.0f ? 1.0f : c2;
      float sum = 0.0f;  // of the lane's q, as it enters the product
      if (a.bf16 || kBits == 4) {
        uint32_t most = 0;  // the largest finite |q|
        const uint32_t inf = a.bf16 ? 0x7F80u : 0x7C00u;
        auto finite = [inf](uint32_t w) { return (w & inf) == inf ? 0u : w & 0x7FFFu; };
#pragma unroll
        for (int p = 0; p < kKc; ++p) {
          const uint32_t w[4] = {q[p].x, q[p].y, q[p].z, q[p].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) most = max(most, max(finite(w[i] & 0xFFFFu), finite(w[i] >> 16)));
        }
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        const float largest = a.bf16 ? from16<true>(static_cast<uint16_t>(most)) : from16<false>(static_cast<uint16_t>(most));
        const int up = most == 0 ? 0 : min(100, 14 - (static_cast<int>(__float_as_uint(largest) >> 23) - 127));
        const float by = sign * __uint_as_float(static_cast<uint32_t>(127 + up) << 23);
        f *= __uint_as_float(static_cast<uint32_t>(127 - up) << 23);
        auto scaled = [&](uint32_t w) {
          const float2 v = a.bf16 ? unpack2<true>(w) : unpack2<false>(w);
          const uint32_t s = pack2<false>(v.x * by, v.y * by);
          const float2 r = unpack2<false>(s);
          sum += r.x + r.y;
          return s;
        };
#pragma unroll
        for (int p = 0; p < kKc; ++p) q[p] = make_uint4(scaled(q[p].x), scaled(q[p].y), scaled(q[p].z), scaled(q[p].w));
      } else if (sign != 1.0f) {
        auto scaled = [sign](uint32_t w) {
          const float2 v = unpack2<false>(w);
          return pack2<false>(v.x * sign, v.y * sign);
        };
#pragma unroll
        for (int p = 0; p < kKc; ++p) q[p] = make_uint4(scaled(q[p].x), scaled(q[p].y), scaled(q[p].z), scaled(q[p].w));
      }
      if constexpr (kBits == 4) {
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
        f *= 0x1p24f;
#pragma unroll
        for (int e = 0; e < 2; ++e) begin[n][e] = __shfl_sync(0xFFFFFFFFu, sum, 4 * (2 * t + e)) * -0x1p-21f;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) fq[n][e] = fmaxf(0x1p-126f, __shfl_sync(0xFFFFFFFFu, f, 4 * (2 * t + e)));
#pragma unroll
      for (int p = 0; p < kKc; ++p) {
        if constexpr (kBits == 4) {  // the nibbles' pairs, the odd ones over 16 (below 2^-25 of the head's largest not exact)
          auto over16 = [](uint32_t w) {
            const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&w), __float2half2_rn(0.0625f));
            return *reinterpret_cast<const uint32_t*>(&h);
          };
          q[p] = make_uint4(__byte_perm(q[p].x, q[p].z, 0x5410), over16(__byte_perm(q[p].x, q[p].z, 0x7632)),
                            __byte_perm(q[p].y, q[p].w, 0x5410), over16(__byte_perm(q[p].y, q[p].w, 0x7632)));
        }
        sq[n][p][lane] = q[p];
      }
    }
    __syncwarp();
    int stage = 0;
    // the lane's rows in a block's place: keys g, g + 8, values 2 t, 2 t + 1, 2 t + 8, 2 t + 9
    uint32_t ka[2], va[4];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      ka[e] = place(g + 8 * e, kKw == 8 ? 2 * t : kKw == 4 ? t : t >> 1) + (kKw == 2 ? 8 * (t & 1) : 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = 2 * t + (e & 1) + 8 * (e >> 1);
      va[e] = 16 * kRow + place(row, kVw == 4 ? g : kVw == 2 ? g >> 1 : g >> 2) + (kVw == 2 ? 8 * (g & 1) : kVw == 1 ? 4 * (g & 3) : 0);
    }
    // The reference is the product `top` that a head's p are 1 at; it moves at `limit`, 2^kMove above.
    float top[kNt][2], limit[kNt][2], back_to[kNt][2];
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        top[n][e] = limit[n][e] = -INFINITY;
        back_to[n][e] = 0.0f;  // -top fq
      }
    // Weights p sv of a head count times wf, at most 2^15; room = 2^15 / wf (0 and 0: none has been seen yet).
    float wf[kNt][2], room[kNt][2];
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) wf[n][e] = room[n][e] = 0.0f;

    for (int tl = tile; tl < tile_end; ++tl) {
      cp_async_wait<kStages - 2>();
      __syncwarp();  // this tile has landed for all lanes, and all have read the one whose stage is next
      const uint32_t there = there_of[0];
#pragma unroll
      for (int i = 0; i + 1 < kStages - 1; ++i) there_of[i] = there_of[i + 1];
      const int next = stage == 0 ? kStages - 1 : stage - 1;
      there_of[kStages - 2] = tl + kStages - 1 < tile_end ? copy(tl + kStages - 1, next) : 0u;
      cp_async_commit();
      const uint32_t from = slots_at + stage * (kRep * kBlock);
      stage = stage == kStages - 1 ? 0 : stage + 1;
      float s[kRep][kNt][4];
#pragma unroll
      for (int r = 0; r < kRep; ++r)
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r][n][e] = kBits == 4 ? begin[n][e & 1] : 0.0f;
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        uint32_t kr[2][kKw];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          read_words<kKw == 8 ? 4 : kKw>(kr[e], from + r * kBlock + ka[e]);
          if constexpr (kKw == 8) read_words<4>(kr[e] + 4, from + r * kBlock + (ka[e] ^ 16u));  // (the other of two chunks)
        }
#pragma unroll
        for (int p = 0; p < kKc; ++p) {
          uint32_t x[2][4];  // of rows g, g + 8: four pairs of codes
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if constexpr (kBits == 8) {
              const uint32_t w0 = kr[e][2 * p] ^ 0x80808080u, w1 = kr[e][2 * p + 1] ^ 0x80808080u;
              x[e][0] = codes8<0>(w0, magic);
              x[e][1] = codes8<1>(w0, magic);
              x[e][2] = codes8<0>(w1, magic);
              x[e][3] = codes8<1>(w1, magic);
            } else {
              const uint32_t w = kr[e][p];
              x[e][0] = key_codes4<0>(w, magic);
              x[e][1] = key_codes4<1>(w, magic);
              x[e][2] = key_codes4<0>(w >> 8, magic);
              x[e][3] = key_codes4<1>(w >> 8, magic);
            }
          }
#pragma unroll
          for (int n = 0; n < kNt; ++n) {
            const uint4 f = reload16(&sq[n][p][lane]);
            mma16816<false>(s[r][n], x[0][0], x[1][0], x[0][1], x[1][1], f.x, f.y);
            mma16816<false>(s[r][n], x[0][2], x[1][2], x[0][3], x[1][3], f.z, f.w);
          }
        }
      }
      const uint32_t counts = counting(tl, there);
      float sv[kRep][2];
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        uint32_t ks[2], vs[2];
        read_words<2>(ks, from + r * kBlock + 32 * kRow + 8 * g);
        read_words<2>(vs, from + r * kBlock + 32 * kRow + 64 + 8 * g);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          sv[r][e] = __uint_as_float(vs[e]);
#pragma unroll
          for (int n = 0; n < kNt; ++n) {
            s[r][n][2 * e] *= __uint_as_float(ks[e]);
            s[r][n][2 * e + 1] *= __uint_as_float(ks[e]);
          }
        }
      }
      if (counts != kAll) {
#pragma unroll
        for (int r = 0; r < kRep; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (!(counts >> (2 * r + e) & 1u)) {
              sv[r][e] = 0.0f;
#pragma unroll
              for (int n = 0; n < kNt; ++n) s[r][n][2 * e] = s[r][n][2 * e + 1] = -INFINITY;
            }
      }
      __syncwarp();
      bool move = false;
#pragma unroll
      for (int r = 0; r < kRep; ++r)
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) move = move || s[r][n][e] > limit[n][e & 1];
      if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = top[n][e];
#pragma unroll
            for (int r = 0; r < kRep; ++r) m = fmaxf(m, fmaxf(s[r][n][e], s[r][n][e + 2]));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
            const float to = m == -INFINITY ? 0.0f : __fmul_rn(-m, fq[n][e]);
            const float alpha = m == top[n][e] ? 1.0f : top[n][e] == -INFINITY ? 0.0f : exp2_fast(__fsub_rn(to, back_to[n][e]));
            top[n][e] = m;
            limit[n][e] = m == -INFINITY ? -INFINITY : m + kMove / fq[n][e];
            back_to[n][e] = to;
            l[n][e] *= alpha;
            // the largest p sv so far follows the reference, and the weights' factor with it: by the power of two
            // above alpha (within what fp32 has), the rest by which o gets smaller is between 1/2 and 1
            float back = alpha;
            if (alpha < 1.0f && room[n][e] > 0.0f) {
              const int r = static_cast<int>(__float_as_uint(room[n][e]) >> 23) - 127;
              const int to_r = max(-105, r + static_cast<int>(__float_as_uint(alpha) >> 23) - 126);
              room[n][e] = __uint_as_float(static_cast<uint32_t>(127 + to_r) << 23);
              wf[n][e] = __uint_as_float(static_cast<uint32_t>(127 + 15 - to_r) << 23);
              back *= __uint_as_float(static_cast<uint32_t>(127 + r - to_r) << 23);
            }
#pragma unroll
            for (int hh = 0; hh < kVc; ++hh)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                o[n][hh][j][e] *= back;
                o[n][hh][j][e + 2] *= back;
              }
          }
      }
      // p into the sums, p sv in s's place
      move = false;
#pragma unroll
      for (int n = 0; n < kNt; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < kRep; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // (rounded as the reference is: one fma would leave half a place of fp32, from 2^31 on more than p has room for)
              const float p = exp2_fast(__fadd_rn(__fmul_rn(s[r][n][2 * e + i], fq[n][i]), back_to[n][i]));
              l[n][i] += p;
              s[r][n][2 * e + i] = p * sv[r][e];
              move = move || fabsf(s[r][n][2 * e + i]) > room[n][i];
            }
      if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float m = 0.0f;
#pragma unroll
            for (int r = 0; r < kRep; ++r) m = fmaxf(m, fmaxf(fabsf(s[r][n][i]), fabsf(s[r][n][i + 2])));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
            if (m > room[n][i]) {
              // the power of two that takes m to 2^10 - 2^11 (within what fp32 has)
              const int e = min(120, max(-110, static_cast<int>(__float_as_uint(m) >> 23) - 127));
              const float was = room[n][i];
              wf[n][i] = __uint_as_float(static_cast<uint32_t>(127 + 10 - e) << 23);
              room[n][i] = __uint_as_float(static_cast<uint32_t>(127 + 5 + e) << 23);
              const float back = was / room[n][i];
#pragma unroll
              for (int hh = 0; hh < kVc; ++hh)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  o[n][hh][j][i] *= back;
                  o[n][hh][j][i + 2] *= back;
                }
            }
          }
      }
#pragma unroll
      for (int r = 0; r < kRep; ++r) {
        uint32_t pw[kNt][kSecond][2];
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {  // rows g, g + 8
            const float w0 = s[r][n][2 * e] * wf[n][0], w1 = s[r][n][2 * e + 1] * wf[n][1];
            const uint32_t hi = pack2<false>(w0, w1);
            const float2 back = unpack2<false>(hi);
            const uint32_t lo = pack2<false>(w0 - back.x, w1 - back.y);
            if constexpr (kPair) {
              pw[n][0][e] = transpose8x8(t < 2 ? hi : lo);
            } else {
              pw[n][0][e] = transpose8x8(hi);
              pw[n][1][e] = transpose8x8(lo);
            }
          }
        uint32_t vr[4][kVw];
#pragma unroll
        for (int e = 0; e < 4; ++e) read_words<kVw>(vr[e], from + r * kBlock + va[e]);
#pragma unroll
        for (int hh = 0; hh < kVc; ++hh) {
          uint32_t x[4][4];  // [j][operand]: dimensions 2 j, 2 j + 1 of positions 2 t, 2 t + 1; 2 t + 8, 2 t + 9
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if constexpr (kBits == 8) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const uint32_t w0 = vr[2 * e][2 * hh + i], w1 = vr[2 * e + 1][2 * hh + i];
                const uint32_t lo = __byte_perm(w0, w1, 0x5140) ^ 0x80808080u, hi = __byte_perm(w0, w1, 0x7362) ^ 0x80808080u;
                x[2 * i][2 * e] = codes8<0>(lo, magic);
                x[2 * i][2 * e + 1] = codes8<1>(lo, magic);
                x[2 * i + 1][2 * e] = codes8<0>(hi, magic);
                x[2 * i + 1][2 * e + 1] = codes8<1>(hi, magic);
              }
            } else {
              const uint32_t w0 = vr[2 * e][hh], w1 = vr[2 * e + 1][hh];
              const uint32_t lo = __byte_perm(w0, w1, 0x5410), hi = __byte_perm(w0, w1, 0x7632);
              x[0][2 * e] = codes4<0>(lo, magic);
              x[0][2 * e + 1] = codes4<1>(lo, magic);
              x[1][2 * e] = codes4<0>(lo >> 8, magic);
              x[1][2 * e + 1] = codes4<1>(lo >> 8, magic);
              x[2][2 * e] = codes4<0>(hi, magic);
              x[2][2 * e + 1] = codes4<1>(hi, magic);
              x[3][2 * e] = codes4<0>(hi >> 8, magic);
              x[3][2 * e + 1] = codes4<1>(hi >> 8, magic);
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < kNt; ++n)
#pragma unroll
              for (int i = 0; i < kSecond; ++i)
                mma16816<false>(o[n][hh][j], x[j][0], x[j][1], x[j][2], x[j][3], pw[n][i][0], pw[n][i][1]);
        }
      }
    }
    cp_async_wait<0>();  // (what is left: empty groups)
    __syncwarp();        // all lanes have read the ring
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        acc.ref[n][i] = __fmul_rn(top[n][i], fq[n][i]);
        const float back = room[n][i] == 0.0f ? 1.0f : room[n][i] * 0x1p-15f;  // 1 / wf
#pragma unroll
        for (int hh = 0; hh < kVc; ++hh)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            o[n][hh][j][i] *= back;
            o[n][hh][j][i + 2] *= back;
          }
      }
    if constexpr (kPair) {
#pragma unroll
      for (int hh = 0; hh < kVc; ++hh)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[0][hh][j][e] += __shfl_down_sync(0xFFFFFFFFu, o[0][hh][j][e], 2);
    }
  }
};

}  // namespace paged
}  // namespace p4q
