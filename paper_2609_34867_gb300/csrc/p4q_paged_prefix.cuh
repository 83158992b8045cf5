// Sequences behind a shared prefix: which group a sequence is in, how the prefix kernel's
// work is dealt, and what it leaves for the kernel of the sequences' own positions.
//
// The rows of a group and key/value head are its n sequences' G query heads over it, in tiles
// of 128; a unit is such a tile, cut into chunks of 128 of the prefix's positions. All chunks in
// one row, group after group, head after head, tile after tile, are dealt to the CTAs in
// consecutive ranges of `share`. A range that begins in the middle of a unit leaves its part of
// that unit's rows with the CTA's number; the range in which a unit begins, with the rows' own
// (parts: [seqs * H] rows, then [grid][128], each dh values, the reference maximum and the sum).
#pragma once

#include "p4q_paged.cuh"

namespace p4q {
namespace paged {

constexpr int kPrefixRows = 128;   // rows of a tile
constexpr int kPrefixChunk = 128;  // positions of a chunk
constexpr int kPartExtra = 4;      // floats of a part beside the values (two of them used)

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

// The group that sequence b is in, -1 if in none: the last one that begins at or before it.
__device__ __forceinline__ int group_of(const PrefixArgs& a, int b) {
  int lo = 0, hi = a.groups;  // group_start[lo] <= b < group_start[hi], if any
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.group_start[mid] <= b)
      lo = mid;
    else
      hi = mid;
  }
  return a.group_start[lo] <= b && b < a.group_start[lo + 1] ? lo : -1;
}

// The positions of sequence b that the prefix kernel sees for it: its group's prefix, or none
// where it is shorter (a row that ended inside the prefix would need values of its own there:
// 0 times an infinite one that others see is NaN). It has them all to itself then, in the pages of the
// group's first sequence.
__device__ __forceinline__ int prefix_seen(const PrefixArgs& a, int b, int len) {
  const int g = group_of(a, b);
  if (g < 0) return 0;
  const int prefix = min(max(a.prefix_lens[g], 0), paged_room(a.kv));
  return len >= prefix ? prefix : 0;
}

__device__ __forceinline__ int row_of(const PrefixArgs& a, int b, int len) {
  const int g = group_of(a, b);
  if (g < 0 || len >= min(max(a.prefix_lens[g], 0), paged_room(a.kv))) return b;
  return min(max(a.group_start[g], 0), a.kv.seqs - 1);
}

__device__ __forceinline__ unsigned long long prefix_share(unsigned long long total, int grid) {
  return max(1ull, (total + grid - 1) / grid);
}

// Adds to head h of sequence b (dimensions d .. d + 3) what the prefix kernel has for it.
__device__ __forceinline__ void add_prefix_parts(const PrefixArgs& a, int b, int h, int d, float& m, float& sum, float4& v) {
  const int g = group_of(a, b);
  if (g < 0) return;
  const Group r = load_group(a, g);
  const int len = a.lens[b];
  if (r.chunks == 0 || len < r.prefix) return;
  const int G = a.H / a.kv.Hkv, row = (b - r.first) * G + h % G;
  const unsigned long long share = prefix_share(a.base[a.groups], a.grid);
  const unsigned long long x = a.base[g] + static_cast<unsigned long long>(h / G * r.tiles + row / kPrefixRows) * r.chunks;
  const int c0 = min(static_cast<int>(x / share), a.grid - 1);
  const int c1 = min(static_cast<int>((x + r.chunks - 1) / share), a.grid - 1);
  const int pitch = a.kv.dh + kPartExtra;
  const float* const first = a.parts + (static_cast<long long>(b) * a.H + h) * pitch;
  const float* const more = a.parts + (static_cast<long long>(a.kv.seqs) * a.H + row % kPrefixRows) * pitch;
  constexpr int kBatch = 8;  // parts on their way together
  for (int c = c0; c <= c1; c += kBatch) {
    float pm[kBatch], pl[kBatch];
    float4 pv[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      pm[i] = -INFINITY;
      pl[i] = 0.0f;
      pv[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (c + i <= c1) {
        const float* p = c + i == c0 ? first : more + static_cast<long long>(c + i) * kPrefixRows * pitch;
        const float2 ml = *reinterpret_cast<const float2*>(p + a.kv.dh);
        pm[i] = ml.x;
        pl[i] = ml.y;
        pv[i] = *reinterpret_cast<const float4*>(p + d);
      }
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) top = fmaxf(top, pm[i]);
    const float f = m == -INFINITY ? 0.0f : exp2_fast(m - top);
    m = top;
    sum *= f;
    v.x *= f;
    v.y *= f;
    v.z *= f;
    v.w *= f;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float e = pm[i] == -INFINITY ? 0.0f : exp2_fast(pm[i] - top);  // (of NaN sums 0 makes NaN)
      sum += pl[i] * e;
      v.x += pv[i].x * e;
      v.y += pv[i].y * e;
      v.z += pv[i].z * e;
      v.w += pv[i].w * e;
    }
  }
}

}  // namespace paged
}  // namespace p4q
