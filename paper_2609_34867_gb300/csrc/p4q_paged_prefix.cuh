// Sequences behind a shared prefix: which group a sequence is in, how the prefix kernel's
// work is dealt, and what it leaves for the kernel of the sequences' own positions.
//
// The rows of a group and key/value head are its n sequences' G query heads over it, in tiles
// of 128; a unit is such a tile, cut into chunks of 128 of the prefix's positions. All chunks in
// one row, group after group, head after head, tile after tile, are dealt to the CTAs in
// consecutive ranges of equal length. A range that begins in the middle of a unit leaves its part of
// that unit's rows with the CTA's number; the range in which a unit begins, with the rows' own
// (parts: [copies][seqs * H] rows, then [grid][128], each dh values, the reference maximum and the sum).
// A unit's rows are few where little is asked of a prefix: then they stand in the tile two or four times and
// each copy takes its share of every chunk's positions (16 rows behind 661 positions x 40 heads: a chunk
// takes about 1.2 us instead of 3).
#pragma once

#include "p4q_paged.cuh"

namespace p4q {
namespace paged {

constexpr int kPrefixRows = 128;   // rows of a tile
constexpr int kPrefixChunk = 128;  // positions of a chunk
constexpr int kPartExtra = 4;      // floats of a part beside the values (two of them used)
constexpr int kCopies = 4;         // of a tile's rows at most
constexpr int kMaxParts = 32;      // ranges that a unit is cut into, about

// Few rows stand in a tile several times, each copy for its share of the positions, with a part of its own.
__device__ __forceinline__ int copies_of(int rows) { return rows <= kPrefixRows / 4 ? 4 : rows <= kPrefixRows / 2 ? 2 : 1; }

struct Group {
  int first, n;       // sequences first .. first + n - 1
  int prefix;         // positions that they share
  int tiles, chunks;  // per key/value head; of the prefix
};

__device__ __forceinline__ int paged_room(const PagedCache& c) {
  return static_cast<int>(min(static_cast<long long>(c.table_cols) << c.page_log2, 1ll << 30));
}

__device__ __forceinline__ Group load_group(const PrefixArgs& a, int g) {
  Group r;
  r.first = min(max(a.group_start[g], 0), a.kv.seqs);
  r.n = min(max(a.group_start[g + 1], r.first), a.kv.seqs) - r.first;
  r.prefix = min(max(a.prefix_lens[g], 0), paged_room(a.kv));
  r.tiles = (r.n * (a.H / a.kv.Hkv) + kPrefixRows - 1) / kPrefixRows;
  r.chunks = (r.prefix + kPrefixChunk - 1) / kPrefixChunk;
  return r;
}

__device__ __forceinline__ unsigned long long group_chunks(const PrefixArgs& a, const Group& r) {
  return static_cast<unsigned long long>(r.tiles) * static_cast<unsigned int>(a.kv.Hkv) * static_cast<unsigned int>(r.chunks);
}

// 64-bit quotients of numbers that mostly fit in 32.
__device__ __forceinline__ unsigned long long quotient(unsigned long long a, unsigned long long b) {
  if (((a | b) >> 32) == 0) return static_cast<unsigned int>(a) / static_cast<unsigned int>(b);
  return a / b;
}

// A range's chunks, of units of `most` at most: a unit's parts are to be few enough that adding them up does not
// take longer than what they save.
__device__ __forceinline__ unsigned long long prefix_share(unsigned long long total, int most, int grid) {
  return max(max(1ull, quotient(total + grid - 1, grid)), static_cast<unsigned long long>((most + kMaxParts - 1) / kMaxParts));
}

// The sum of x over this lane and those before it.
__device__ __forceinline__ unsigned long long scan_add(unsigned long long x) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long v = __shfl_up_sync(0xFFFFFFFFu, x, d);
    if ((threadIdx.x & 31) >= d) x += v;
  }
  return x;
}

// What lies in front of sequence b's own positions (found by a whole warp).
struct PrefixOf {
  int g = -1;                    // its group, -1: none, or one whose prefix is longer than the sequence (a row that
                                 // ended inside the prefix would need values of its own there: 0 times an infinite
                                 // one that others see is NaN) and which it has to itself then
  Group r = {};
  int from = 0;                  // its first own position
  int row;                       // of the page table, for these: the group's first where it has all to itself
  unsigned long long begin = 0;  // the chunks before its group (of up to 32 groups; else base[g], once the prefix kernel has ended)
  __device__ __forceinline__ PrefixOf(const PrefixArgs& a, int b, int len) : row(b) {
    if (a.groups <= 32) {  // a lane each
      const int lane = threadIdx.x & 31;
      Group gr = {};
      if (lane < a.groups) gr = load_group(a, lane);
      __syncwarp();
      const unsigned long long n = group_chunks(a, gr), upto = scan_add(n);
      const uint32_t in = __ballot_sync(0xFFFFFFFFu, gr.first <= b && b < gr.first + gr.n);
      if (in != 0) {
        g = __ffs(in) - 1;
        r.first = __shfl_sync(0xFFFFFFFFu, gr.first, g);
        r.n = __shfl_sync(0xFFFFFFFFu, gr.n, g);
        r.prefix = __shfl_sync(0xFFFFFFFFu, gr.prefix, g);
        r.tiles = __shfl_sync(0xFFFFFFFFu, gr.tiles, g);
        r.chunks = __shfl_sync(0xFFFFFFFFu, gr.chunks, g);
        begin = __shfl_sync(0xFFFFFFFFu, upto - n, g);
      }
    } else {  // the last one that begins at or before it
      int lo = 0, hi = a.groups;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.group_start[mid] <= b)
          lo = mid;
        else
          hi = mid;
      }
      r = load_group(a, lo);
      if (r.first <= b && b < r.first + r.n) g = lo;
    }
    if (g >= 0 && len < r.prefix) {
      row = r.first;
      g = -1;
    }
    if (g >= 0) from = r.prefix;
    if (g >= 0 && r.chunks == 0) g = -1;
  }
};

}  // namespace paged
}  // namespace p4q
