// The draw of one token from each row of logits: temperature, top-k, top-p and
// min-p with a given uniform number.
//
// Weights are integers (2^31 exp(-d) rounded), so that their sums are exact and
// the drawn token depends on no order of summation, hence on no split of the
// row either. The kept tokens are a head of the row in the order "falling logit,
// then rising index"; each cut is the last token of that head.
//
// A cluster of CTAs takes a row; its logits are read once and stay in shared
// memory, a slice of the row in each CTA.
// A cut is found as follows. A histogram over d in steps of 1 / 92 (counts for
// top-k, weights for top-p) covers every token whose weight is not 0 (2^31 e^-d
// rounds to 0 past d = 22.2; those come last and are never drawn, so they take
// no part). Every CTA gets the sums of all CTAs' groups of 32 bins, one warp of it
// finds the group and, from the CTAs' bins of that, the bin in which the wanted
// sum is reached. The bin's tokens, mostly a few, are gathered in every CTA and
// ranked, a share of them by each. (A scan divided among the CTAs and a ranking by
// one thread per token took 30 k cycles where this takes 7.) Bins
// of more tokens than the lists hold are
// divided again by the logits' ordered bit patterns, at most three times (11 of 32
// bits each); a bin of equal logits is cut by index.
// Mostly few tokens can be kept at all: up to the bin of a top-k or top-p cut, or
// those that pass a min-p. Up to 512 of them go to the cluster's first CTA, which
// sorts them and makes the cuts and the draw on that list alone. A top-k of up to 256
// looks for them with a histogram of the threads' largest logits instead of all
// (a thread then looks through its own if its largest is in reach: 256 x 131072 fp32
// 96 us to 78, 64 x 32000 fp16 11.4 to 10.0). What follows is for the rest:
// The draw: kept weights per CTA (behind a top-p cut they are known from the
// histogram) and their prefix over the cluster; then the one CTA that contains the
// drawn number finds the warp (a warp's tokens are consecutive), and that
// warp walks its tokens.
//
// Bound: phases between barriers of the CTA and the cluster, at two CTAs of 512
// threads per SM, and 25 (a small top-k) to 110 instructions per logit; HBM is at 2 TB/s at
// most. us: 256 x 131072 fp32 without cuts 68, top-k 78, with top-p 78, min-p 65, largest logit only
// 38, top-p of thousands of tokens 190; 64 x 32000 fp16 8.2, 10.0, 10.1, 11.8, 3.9, 20 - 22; one row
// 5.7, 8.2, 8.4, 6.9, 2.9, 13.7. (The loops over a thread's logits are not unrolled: 150 KB of
// code instead of 217, and no slower.)
#include <climits>
#include <cuda_runtime.h>

#include <type_traits>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048;
constexpr float kBinScale = 92.0f;  // 2047 / 92 = 22.25 > 22.18 = ln(2^32): a token past the bins has weight 0
constexpr int kList = 512;          // tokens of a bin that are ranked, at most
constexpr int kOwn = 256;           // of one CTA

constexpr int kGroups = kBins / 32;
constexpr int kPairs = 128;         // candidates that are compared pairwise, at most
constexpr int kCand = 768;          // places for candidates, each CTA a part of them
constexpr float kNear = 8.0f;       // a min-p of at least e^-8 mostly leaves few tokens

struct Shared {
  uint32_t lo[kBins], hi[kBins];  // counts, or the weights' low and high 16 bits
  u64 own[kOwn];      // the CTA's tokens of a bin: key, complement of the index
  union {
    u64 cand[kCand];  // (of the cluster's first CTA) candidates, each CTA's from its part's start
    struct {
      u64 list[kList];  // the cluster's tokens of the bin
      uint32_t weight[kList];
    };
  };
  u64 warp_sum[kWarps];
  // values of each CTA of the cluster, written by it
  u64 group[kMaxCluster][kGroups];  // its sums over 32 bins
  u64 mass[kMaxCluster];
  uint32_t max_key[kMaxCluster], first_max[kMaxCluster], cand_n[kMaxCluster], own_n[kMaxCluster], key_min[kMaxCluster],
      key_max[kMaxCluster];
  u64 need, total, draw;
  u64 cut;                        // the last kept token
  uint32_t bin, sent, n, kmin, kmax;  // candidates sent; of the CTA's list: its length, smallest and largest key
  uint32_t red[kWarps];
  uint32_t param[5];              // the row's temperature, top-k, top-p, min-p and uniform number
};

__device__ __forceinline__ float float_of_key(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ u64 ld_cluster_u64(uint32_t a) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ void st_shared_cluster_u64(uint32_t a, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}

__device__ __forceinline__ u64 warp_add(u64 v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

__device__ __forceinline__ u64 warp_scan(u64 v) {  // inclusive
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 u = __shfl_up_sync(0xFFFFFFFFu, v, d);
    if ((threadIdx.x & 31) >= d) v += u;
  }
  return v;
}

template <int kType>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleArgs a, const int steps) {
  constexpr int kSize = kType == 2 ? 4 : 2;
  extern __shared__ __align__(16) float4 xs[];  // [kWarps][steps][32] the CTA's logits
  __shared__ Shared s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cs = static_cast<int>(cluster_nctarank()), rank = static_cast<int>(cluster_ctarank());
  const int n = static_cast<int>(blockIdx.x) / cs, V = a.vocab;
  auto sync_all = [&]() {
    if (cs > 1) cluster_sync();
    else __syncthreads();
  };
  // The variable in every CTA of the cluster: by one thread, or by a warp's lanes.
  auto put32 = [&](uint32_t* p, uint32_t v) {
#pragma unroll 1
    for (int r = 0; r < cs; ++r) st_shared_cluster_u32(mapa_shared(smem_u32(p), r), v);
  };
  auto put64 = [&](u64* p, u64 v) {
    put32(reinterpret_cast<uint32_t*>(p), static_cast<uint32_t>(v));
    put32(reinterpret_cast<uint32_t*>(p) + 1, static_cast<uint32_t>(v >> 32));
  };
  auto put64_lanes = [&](u64* p, u64 v) {
    if (lane < cs) st_shared_cluster_u64(mapa_shared(smem_u32(p), lane), v);
  };
  auto put32_lanes = [&](uint32_t* p, uint32_t v) {
    if (lane < cs) st_shared_cluster_u32(mapa_shared(smem_u32(p), lane), v);
  };

  if (cs > 1) cluster_begun_arrive();
  pdl_wait();
  pdl_launch_dependents();

  // The row from the 16-byte boundary at or before it: element e there is token
  // e - skip. A warp takes steps x 128 consecutive elements and keeps them to
  // itself: no barrier stands between its stores here and its passes.
  const char* row = static_cast<const char*>(a.logits) + n * a.ld * kSize;
  const int skip = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15u) / kSize;
  const int end = V + skip;
  row -= skip * kSize;
  const int w0 = (rank * kWarps + warp) * steps * 128;  // the warp's first element
  // What is needed later, while the row is under way: the row's parameters, an empty histogram
  uint32_t param = 0;
  if (tid < 5) {
    const void* const from = tid == 0 ? static_cast<const void*>(a.temperature)
                             : tid == 1 ? static_cast<const void*>(a.top_k)
                             : tid == 2 ? static_cast<const void*>(a.top_p)
                             : tid == 3 ? static_cast<const void*>(a.min_p)
                                        : static_cast<const void*>(a.u);
    param = from ? static_cast<const uint32_t*>(from)[n] : tid == 0 || tid == 2 ? 0x3F800000u : 0u;
  }
  auto empty = [&]() {  // the histogram and the lists
    for (int i = tid; i < kBins; i += kThreads) s.lo[i] = s.hi[i] = 0;
    if (tid == 0) {
      s.sent = 0;
      s.n = 0;
      s.kmin = 0xFFFFFFFFu;
      s.kmax = 0;
    }
  };
  empty();
  bool is_empty = true;
  float4* const mine4 = xs + warp * steps * 32;
  auto clean = [](float v) { return fmaxf(v, -INFINITY); };  // NaN counts as -inf
  float mx = -INFINITY;
  // 16 bytes of the row from element e on, -inf where it has none
  auto edge = [&](int e) {
    uint32_t raw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (kType == 2) {
        raw[j] = e + j >= skip && e + j < end ? reinterpret_cast<const uint32_t*>(row)[e + j] : 0xFF800000u;
      } else {
        constexpr uint32_t kNone = kType == 1 ? 0xFF80u : 0xFC00u;
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
        const int m = e + 2 * j;
        const uint32_t l = m >= skip && m < end ? p[m] : kNone;
        const uint32_t h = m + 1 >= skip && m + 1 < end ? p[m + 1] : kNone;
        raw[j] = l | (h << 16);
      }
    }
    return make_uint4(raw[0], raw[1], raw[2], raw[3]);
  };
  // load k of this lane: 16 bytes, 4 or 8 logits
  auto keep = [&](int k, uint4 raw) {
    if (kType == 2) {
      const float4 v = make_float4(clean(__uint_as_float(raw.x)), clean(__uint_as_float(raw.y)),
                                   clean(__uint_as_float(raw.z)), clean(__uint_as_float(raw.w)));
      mine4[k * 32 + lane] = v;
      mx = fmaxf(fmaxf(fmaxf(mx, v.x), fmaxf(v.y, v.z)), v.w);
    } else {
      const uint32_t r[4] = {raw.x, raw.y, raw.z, raw.w};
      float f[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = unpack2<kType == 1>(r[j]);
        f[2 * j] = clean(v.x);
        f[2 * j + 1] = clean(v.y);
        mx = fmaxf(mx, fmaxf(f[2 * j], f[2 * j + 1]));
      }
      mine4[(k * 32 + lane) * 2] = make_float4(f[0], f[1], f[2], f[3]);
      mine4[(k * 32 + lane) * 2 + 1] = make_float4(f[4], f[5], f[6], f[7]);
    }
  };
  constexpr int kPer = 16 / kSize;  // logits per load
  const int loads = steps * 128 / (32 * kPer);
  const uint4* const src = reinterpret_cast<const uint4*>(row + static_cast<size_t>(w0) * kSize) + lane;
  if (w0 >= skip && w0 + steps * 128 <= end) {  // (the warp alike) all inside the row: eight loads in flight
    int k = 0;
    for (; k + 8 <= loads; k += 8) {
      uint4 raw[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) raw[j] = src[(k + j) * 32];
#pragma unroll
      for (int j = 0; j < 8; ++j) keep(k + j, raw[j]);
    }
    for (; k + 2 <= loads; k += 2) {
      const uint4 r0 = src[k * 32], r1 = src[(k + 1) * 32];
      keep(k, r0);
      keep(k + 1, r1);
    }
    for (; k < loads; ++k) keep(k, src[k * 32]);
  } else {  // four, then the 16 bytes that the row begins or ends in (one load after the other, with those
            // in their places: 256 x 131071 fp32 58 us instead of 41, of 131072 38)
    constexpr uint32_t kNone = kType == 2 ? 0xFF800000u : kType == 1 ? 0xFF80FF80u : 0xFC00FC00u;
    for (int k = 0; k < loads; k += 4) {
      uint4 raw[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = w0 + ((k + j) * 32 + lane) * kPer;
        raw[j] = make_uint4(kNone, kNone, kNone, kNone);
        if (k + j < loads && e >= skip && e + kPer <= end) raw[j] = src[(k + j) * 32];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k + j < loads) keep(k + j, raw[j]);
    }
#pragma unroll 1
    for (int x = 0; x < 2; ++x) {
      const int e = x == 0 ? 0 : (end - 1) / kPer * kPer, at = (e - w0) / kPer;
      if (e >= w0 && at < loads * 32 && at % 32 == lane && (e < skip || e + kPer > end)) keep(at / 32, edge(e));
    }
  }
  if (tid < 5) s.param[tid] = param;
  const float own_mx = mx;  // this lane's
  __syncwarp();
  // f(logit, token) for this lane's four tokens of a step; for all of them
  const int i0 = w0 + lane * 4 - skip;
  auto four = [&](int st, auto&& f) {
    const float4 v = mine4[st * 32 + lane];
    const int i = i0 + st * 128;
    f(v.x, i);
    f(v.y, i + 1);
    f(v.z, i + 2);
    f(v.w, i + 3);
  };
  auto each = [&](auto&& f) {
#pragma unroll 1
    for (int st = 0; st < steps; ++st) four(st, f);
  };
  auto key_of = [](float v) { return float_order_key(v + 0.0f); };  // (-0 as +0)

  // the row's largest logit
  {
    const uint32_t k = __reduce_max_sync(0xFFFFFFFFu, key_of(mx));
    if (lane == 0) s.red[warp] = k;
    __syncthreads();
    if (cs > 1) cluster_begun_wait();
    if (warp == 0) {
      const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, s.red[lane & (kWarps - 1)]);
      put32_lanes(&s.max_key[rank], all);
    }
    sync_all();
    uint32_t best = s.max_key[0];
    for (int r = 1; r < cs; ++r) best = max(best, s.max_key[r]);
    mx = float_of_key(best);
  }
  if (mx == -INFINITY) {
    if (rank == 0 && tid == 0) {
      a.token[n] = -1;
      if (a.logprob) a.logprob[n] = -INFINITY;
    }
    return;
  }
  const float temp = __uint_as_float(s.param[0]);
  if (!(temp > 0.0f)) {  // the first of the largest
    uint32_t first = 0xFFFFFFFFu;
    each([&](float v, int i) {
      if (v == mx) first = min(first, static_cast<uint32_t>(i));
    });
    first = __reduce_min_sync(0xFFFFFFFFu, first);
    if (lane == 0) s.red[warp] = first;  // (the maxima there were read before the last barrier)
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) first = min(first, s.red[w]);
      st_shared_cluster_u32(mapa_shared(smem_u32(&s.first_max[rank]), 0), first);
    }
    sync_all();
    if (rank == 0 && tid == 0) {
      for (int r = 0; r < cs; ++r) first = min(first, s.first_max[r]);
      a.token[n] = static_cast<int32_t>(first);
      if (a.logprob) a.logprob[n] = 0.0f;
    }
    return;
  }

  // (T = inf: not 0, so that a logit of -inf stays infinitely far)
  const float inv_t = fmaxf(1.0f / temp, 1.17549435e-38f);
  // (the largest itself: 0, also where the product is NaN: of infinite logits, of a denormal T)
  auto dist = [&](float v) { return fmaxf((mx - v) * inv_t, 0.0f); };
  auto weight = [&](float d) { return __float2uint_rn(expf(-d) * 2147483648.0f); };
  // the bin of d = dist(v): rounded to an integer behind 2^23 (the largest logit itself: 0, as in dist)
  constexpr float kBinBase = 8388608.0f;
  // (finite, so that differences as small as a tiny T have bins: smaller steps of d then)
  const float bin_scale = fminf(inv_t * kBinScale, 3.402823466e38f);
  auto d_bin = [&](float v) { return fmaxf(fmaf(mx - v, bin_scale, kBinBase), kBinBase); };
  float cut_x = -INFINITY;  // the last kept token
  int cut_i = INT_MAX;
  auto keeps = [&](float v, int i) { return v >= cut_x && !(v == cut_x && i > cut_i); };
  u64 cta_mass = 0;  // the kept weights of the CTA, where known
  bool known = false;

  // Sends the tokens of a step's four logits with `in` to the first CTA's candidates
  // (the CTA's own part of them, as far as it goes; s.sent counts all).
  const int room = kCand / cs;
  auto send = [&](const float (&v)[4], int i, const bool (&in)[4]) {
    if (!__any_sync(0xFFFFFFFFu, in[0] || in[1] || in[2] || in[3])) return;
    // too many already (by one lane's reading, as other warps count on)
    if (__shfl_sync(0xFFFFFFFFu, *reinterpret_cast<volatile uint32_t*>(&s.sent), 0) > static_cast<uint32_t>(room)) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t with = __ballot_sync(0xFFFFFFFFu, in[j]);
      if (with == 0) continue;
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&s.sent, static_cast<uint32_t>(__popc(with)));
      at = __shfl_sync(0xFFFFFFFFu, at, 0) + static_cast<uint32_t>(__popc(with & ((1u << lane) - 1u)));
      if (in[j] && at < static_cast<uint32_t>(room))
        st_shared_cluster_u64(mapa_shared(smem_u32(&s.cand[rank * room + at]), 0),
                              static_cast<u64>(key_of(v[j])) << 32 | static_cast<uint32_t>(~(i + j)));
    }
  };
  // How many candidates there are, or 0 if they do not all have a place (the counts are there).
  auto candidates = [&]() -> uint32_t {
    uint32_t all = 0, most = 0;
    for (int r = 0; r < cs; ++r) {
      all += s.cand_n[r];
      most = max(most, s.cand_n[r]);
    }
    return all <= kList && most <= static_cast<uint32_t>(room) ? all : 0u;
  };
  const int top_k = static_cast<int>(s.param[1]);
  const float top_p = __uint_as_float(s.param[2]);
  float min_p = __uint_as_float(s.param[3]);
  min_p = min_p > 0.0f ? fminf(min_p, 1.0f) : 0.0f;  // (NaN: none)
  // past d_max exp(-d) < min_p for certain (weights are 0 past 22.2)
  const float d_max = fminf(min_p > 0.0f ? 1e-5f - 1.000001f * logf(min_p) : 23.0f, 23.0f);
  const bool by_k = top_k > 0 && top_k < V, by_p = top_p < 1.0f;
  auto sum_cta = [&](u64 v) -> u64 {  // over the CTA's threads
    v = warp_add(v);
    __syncthreads();
    if (lane == 0) s.warp_sum[warp] = v;
    __syncthreads();
    u64 all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all += s.warp_sum[w];
    return all;
  };
  // Sorts a value of each of the first `size` threads (a multiple of 32, up to kList), falling, all threads calling;
  // `count` values are not 0, and no two of these alike. The warps sort theirs, then each value's place is its own
  // warp's and what searches in the others' find larger.
  auto sort = [&](u64 v, uint32_t size, uint32_t count) -> u64 {
#pragma unroll 1
    for (uint32_t k = 2; k <= 32; k <<= 1)
#pragma unroll 1
      for (uint32_t j = k >> 1; j > 0; j >>= 1) {
        const u64 other = __shfl_xor_sync(0xFFFFFFFFu, v, j);
        const bool larger = ((lane & k) == 0) == ((lane & j) == 0);
        v = larger == (other > v) ? other : v;
      }
    s.list[tid] = v;
    __syncthreads();
    uint32_t place = static_cast<uint32_t>(lane);
    if (v != 0) {
#pragma unroll 4
      for (uint32_t w = 0; w < size; w += 32) {
        const u64* const in = s.list + w;
        uint32_t more = 0;
#pragma unroll
        for (uint32_t step = 16; step > 0; step >>= 1) more += in[more + step - 1] > v ? step : 0u;
        more += in[more] > v ? 1u : 0u;
        place += w == static_cast<uint32_t>(warp) * 32 ? 0u : more;
      }
    }
    __syncthreads();
    if (v != 0) s.list[place] = v;
    __syncthreads();
    return static_cast<uint32_t>(tid) < count ? s.list[tid] : 0ull;
  };
  // Inclusive scan over the CTA's threads; *all: the sum.
  auto scan_cta = [&](u64 v, u64* all) -> u64 {
    u64 to = warp_scan(v);
    __syncthreads();
    if (lane == 31) s.warp_sum[warp] = to;
    __syncthreads();
    u64 sum = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) to += s.warp_sum[w];
      sum += s.warp_sum[w];
    }
    *all = sum;
    return to;
  };
  static_assert(kList == kThreads, "a candidate per thread");
  // The cuts and the draw on the `found` candidates, by the first CTA. with_k: they are the first top_k
  // tokens and some after these; else s.total is the sum of the weights that a top-p is a share of.
  // Up to 128 are compared pairwise (kThreads / size lanes per token), more are sorted (200 of 64 x 32000 fp16
  // 14.2 us, pairwise 21.5, by a bitonic sort of all 16.4; 400: 22.6 and 21.7). Likewise the kept ones, for the
  // draw by index.
  auto finish = [&](uint32_t found, bool with_k) {
    uint32_t size = 32;
    while (size < found) size <<= 1;
    const bool pairs = size <= kPairs;
    const int ways = pairs ? kThreads / static_cast<int>(size) : 1;  // 4 .. 16 neighbouring lanes
    const uint32_t at = static_cast<uint32_t>(tid / ways), way = static_cast<uint32_t>(tid % ways);
    u64 t = 0;  // (no token: below every token)
    if (at < found) {
      int r = 0;
      uint32_t j = at;
      while (j >= s.cand_n[r]) j -= s.cand_n[r++];
      t = s.cand[r * room + j];
    }
    __syncthreads();  // (the list lies in the same place)
    if (!pairs) t = sort(t, size, found);
    const bool real = at < found;
    const float e = real ? expf(-dist(float_of_key(static_cast<uint32_t>(t >> 32)))) : 0.0f;
    const uint32_t w = __float2uint_rn(e * 2147483648.0f);
    uint32_t place = at;  // among the candidates
    u64 before = 0;       // the weights before it
    auto sum_lanes = [](u64 v, int lanes) {  // over neighbouring lanes
#pragma unroll 1
      for (int x = 1; x < lanes; x <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, x);
      return v;
    };
    if (pairs) {
      if (way == 0) {
        s.list[at] = t;
        s.weight[at] = w;
      }
      __syncthreads();
      uint32_t c = 0;
      for (uint32_t j = way; j < found; j += ways)
        if (s.list[j] > t) {
          ++c;
          before += s.weight[j];
        }
      place = static_cast<uint32_t>(sum_lanes(c, ways));
      before = sum_lanes(before, ways);
    }
    const bool in_k = real && !(with_k && place >= static_cast<uint32_t>(top_k));
    if (by_p) {
      u64 sum = before + w;  // (of the last of the first top_k: theirs)
      bool last = way == 0 && place == min(static_cast<uint32_t>(top_k), found) - 1;
      if (!pairs) {
        before = scan_cta(in_k ? w : 0u, &sum) - w;
        last = tid == 0;
      }
      if (with_k ? last : tid == 0) {  // (64-bit floating point is slow: once)
        const double part = ceil(static_cast<double>(top_p) * static_cast<double>(with_k ? sum : s.total));
        s.need = part < 1.0 ? 1ull : static_cast<u64>(part);
      }
      __syncthreads();
    }
    const bool is_kept = in_k && w > 0 && !(e < min_p) && (!by_p || before < s.need);
    // The draw: the kept tokens are the first ones; by index: its complement, and the weight.
    const uint32_t kept = static_cast<uint32_t>(__syncthreads_count(is_kept && way == 0));  // (the list has been read)
    u64 mine = is_kept ? static_cast<u64>(static_cast<uint32_t>(t)) << 32 | w : 0ull;
    u64 upto = 0, total = 0;  // the kept weights up to this token, all
    uint32_t key = 0;         // this token's logit
    bool leader = true;
    if (kept <= kPairs) {
      if (is_kept && way == 0) {
        s.list[place] = mine;
        s.own[place] = t;
      }
      int per = kThreads / 32;  // lanes per token
      while (kThreads / per < static_cast<int>(kept)) per >>= 1;
      __syncthreads();
      const uint32_t to = static_cast<uint32_t>(tid / per), first = static_cast<uint32_t>(tid % per);
      mine = to < kept ? s.list[to] : 0ull;
      key = to < kept ? static_cast<uint32_t>(s.own[to] >> 32) : 0u;
      leader = first == 0;
      for (uint32_t j = first; j < kept; j += per) {
        const u64 x = s.list[j];
        total += static_cast<uint32_t>(x);
        if (x >= mine) upto += static_cast<uint32_t>(x);
      }
      upto = sum_lanes(upto, per);
      total = sum_lanes(total, per);
    } else {
      mine = sort(mine, size, kept);
      upto = scan_cta(static_cast<uint32_t>(mine), &total);
    }
    if (tid == 0) {
      const double want = floor(static_cast<double>(__uint_as_float(s.param[4])) * static_cast<double>(total));
      const u64 r = want > 0.0 ? static_cast<u64>(fmin(want, 9.0e15)) : 0ull;
      s.draw = min(r, total - 1);
    }
    __syncthreads();
    const u64 r = s.draw;
    if (leader && upto - static_cast<uint32_t>(mine) <= r && r < upto) {
      const int i = static_cast<int>(~static_cast<uint32_t>(mine >> 32));
      a.token[n] = i;
      if (a.logprob) {
        float x = float_of_key(key);
        if (kept > kPairs) {  // (sorted without it)
          const void* p = row + static_cast<size_t>(i + skip) * kSize;
          x = kType == 2 ? *static_cast<const float*>(p) : from16<kType == 1>(*static_cast<const uint16_t*>(p));
        }
        a.logprob[n] = -dist(x) - logf(static_cast<float>(static_cast<double>(total) * 4.656612873077393e-10));
      }
    }
  };

  // Shortens the kept head: to `need` tokens, or (by_mass) to the first tokens
  // whose weights reach ceil(share * the kept weights' sum). Where the kept tokens are few, it only finds
  // found_n candidates.
  uint32_t found_n = 0;  // candidates that the first CTA draws one of
  bool found_k = false;
  auto shorten = [&](auto mass_c, u64 need, float share) {
    constexpr bool by_mass = decltype(mass_c)::value;
    uint32_t key_lo = 0, key_hi = 0;
    int shift = 0;
    u64 below = 0;  // (by_mass) the CTA's weights before the bin
    // Of the first `need` tokens mostly a histogram of the lanes' largest logits alone will do: up to the bin in
    // which `need` lanes are reached there are as many tokens or more, and few more while the lanes are many.
    bool lanes = !by_mass && need <= kList / 2 && need <= static_cast<u64>(cs) * (kThreads / 2);
    for (int level = 0;;) {
      if (!is_empty) {
        empty();
        __syncthreads();
      }
      is_empty = false;
      // the bin of a token behind kBinBase's bit pattern (falling logits have rising bins); past the bins: larger
      auto bin_of = [&](float v) -> int {
        if (level == 0) return __float_as_int(d_bin(v));
        const uint32_t k = key_of(v);
        return k >= key_lo && k <= key_hi ? __float_as_int(kBinBase) + static_cast<int>((key_hi - k) >> shift) : INT_MAX;
      };
      if (lanes) {
        const uint32_t bin = static_cast<uint32_t>(__float_as_int(d_bin(own_mx)) - __float_as_int(kBinBase));
        if (bin < kBins) atomicAdd(&s.lo[bin], 1u);
      }
#pragma unroll 1
      for (int st = lanes ? steps : 0; st < steps; ++st) {
        const float4 v4 = mine4[st * 32 + lane];
        const float v[4] = {v4.x, v4.y, v4.z, v4.w};
        uint32_t bin[4], w[4];
        bool any = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bin[j] = static_cast<uint32_t>(bin_of(v[j]) - __float_as_int(kBinBase));
          if (by_mass && !keeps(v[j], i0 + st * 128 + j)) bin[j] = kBins;
          any = any || bin[j] < kBins;
        }
        if (!any) continue;
        if (by_mass) {
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = weight(dist(v[j]));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (bin[j] >= kBins) continue;
          if (by_mass) {
            atomicAdd(&s.lo[bin[j]], w[j] & 0xFFFFu);
            if (w[j] >> 16) atomicAdd(&s.hi[bin[j]], w[j] >> 16);
          } else {
            atomicAdd(&s.lo[bin[j]], 1u);
          }
        }
      }
      __syncthreads();
      // sums of 32 bins each, to every CTA
#pragma unroll
      for (int j = 0; j < kGroups / kWarps; ++j) {
        const int g = warp * (kGroups / kWarps) + j;
        // (32 bits hold them: a CTA has at most 36864 tokens of less than 2^16 each)
        u64 v = __reduce_add_sync(0xFFFFFFFFu, s.lo[g * 32 + lane]);
        if (by_mass) v += static_cast<u64>(__reduce_add_sync(0xFFFFFFFFu, s.hi[g * 32 + lane])) << 16;
        put64_lanes(&s.group[rank][g], v);
      }
      sync_all();
      if (warp == 0) {  // the group, then the bin in which the sum is reached
        u64 g0 = 0, g1 = 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
          if (r < cs) {
            g0 += s.group[r][2 * lane];
            g1 += s.group[r][2 * lane + 1];
          }
        u64 upto = warp_scan(g0 + g1);
        const u64 total = __shfl_sync(0xFFFFFFFFu, upto, 31);
        u64 want = need;
        if (by_mass && level == 0) {
          const double part = ceil(static_cast<double>(share) * static_cast<double>(total));
          want = part < 1.0 ? 1ull : static_cast<u64>(part);
        }
        // (not reached at all: the last group, and the caller goes by `total`)
        const uint32_t there = __ballot_sync(0xFFFFFFFFu, upto >= want);
        const int at_lane = there ? __ffs(there) - 1 : 31;
        const u64 before = upto - g0 - g1;
        const bool second = before + g0 < want;
        const int g = __shfl_sync(0xFFFFFFFFu, 2 * lane + (second ? 1 : 0), at_lane);
        want -= __shfl_sync(0xFFFFFFFFu, second ? before + g0 : before, at_lane);
        u64 v = 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
          if (r < cs) {
            v += ld_cluster_u32(mapa_shared(smem_u32(&s.lo[g * 32 + lane]), r));
            if (by_mass) v += static_cast<u64>(ld_cluster_u32(mapa_shared(smem_u32(&s.hi[g * 32 + lane]), r))) << 16;
          }
        upto = warp_scan(v);
        if (upto >= want && upto - v < want) {
          s.bin = static_cast<uint32_t>(g * 32 + lane);
          s.need = want - (upto - v);
        }
        if (lane == 0) s.total = total;
      }
      __syncthreads();
      const int cut_bin = static_cast<int>(s.bin);
      if (!by_mass && level == 0 && s.total <= need) {
        sync_all();  // (the CTAs' bins and sums have been read)
        if (!lanes) return;  // every token that may be drawn is among the first `need`
        lanes = false;
        continue;
      }
      const bool few = level == 0 && (by_mass || need <= kList);  // the tokens up to the bin may be few
      const int cut_bits = __float_as_int(kBinBase) + cut_bin;
      if (lanes) {
        if (__float_as_int(d_bin(own_mx)) <= cut_bits) {
          for (int st = 0; st < steps; ++st) {  // the logits that this lane loaded
            const int at4 = kType == 2 ? st * 32 + lane : ((st >> 1) * 32 + lane) * 2 + (st & 1);
            const float4 v4 = mine4[at4];
            const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (__float_as_int(d_bin(v[j])) > cut_bits) continue;
              const uint32_t at = atomicAdd(&s.sent, 1u);
              if (at < static_cast<uint32_t>(room))
                st_shared_cluster_u64(mapa_shared(smem_u32(&s.cand[rank * room + at]), 0),
                                      static_cast<u64>(key_of(v[j])) << 32 |
                                          static_cast<uint32_t>(~(w0 - skip + at4 * 4 + j)));
            }
          }
        }
        __syncthreads();
        if (warp == 0) put32_lanes(&s.cand_n[rank], s.sent);
        sync_all();
        found_n = candidates();
        found_k = true;
        if (found_n > 0) return;
        sync_all();  // (the counts have been read)
        lanes = false;
        continue;
      }
      need = s.need;
      // The bin's tokens of this CTA; those up to it to the first CTA.
      uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
      const bool none = level == 0 && !__any_sync(0xFFFFFFFFu, __float_as_int(d_bin(own_mx)) <= cut_bits);
#pragma unroll 1
      for (int st = none ? steps : 0; st < steps; ++st) {
        const float4 v4 = mine4[st * 32 + lane];
        const float v[4] = {v4.x, v4.y, v4.z, v4.w};
        const int bits[4] = {bin_of(v[0]), bin_of(v[1]), bin_of(v[2]), bin_of(v[3])};
        if (!__any_sync(0xFFFFFFFFu, min(min(bits[0], bits[1]), min(bits[2], bits[3])) <= cut_bits)) continue;
        bool in[4], at_cut[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          in[j] = bits[j] <= cut_bits && (!by_mass || keeps(v[j], i0 + st * 128 + j));
          at_cut[j] = in[j] && bits[j] == cut_bits;
        }
        if (few) send(v, i0 + st * 128, in);
        if (!__any_sync(0xFFFFFFFFu, at_cut[0] || at_cut[1] || at_cut[2] || at_cut[3])) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t with = __ballot_sync(0xFFFFFFFFu, at_cut[j]);
          if (with == 0) continue;
          uint32_t at = 0;
          if (lane == 0) at = atomicAdd(&s.n, static_cast<uint32_t>(__popc(with)));
          at = __shfl_sync(0xFFFFFFFFu, at, 0) + static_cast<uint32_t>(__popc(with & ((1u << lane) - 1u)));
          if (at_cut[j]) {
            const uint32_t key = key_of(v[j]);
            kmin = min(kmin, key);
            kmax = max(kmax, key);
            if (at < kOwn) s.own[at] = static_cast<u64>(key) << 32 | static_cast<uint32_t>(~(i0 + st * 128 + j));
          }
        }
      }
      if (kmin <= kmax) {
        atomicMin(&s.kmin, kmin);
        atomicMax(&s.kmax, kmax);
      }
      if (by_mass) {
        u64 sum = 0;
        for (int i = tid; i < cut_bin; i += kThreads) sum += s.lo[i] + (static_cast<u64>(s.hi[i]) << 16);
        sum = warp_add(sum);
        if (lane == 0) s.warp_sum[warp] = sum;
      }
      __syncthreads();
      if (by_mass) {
#pragma unroll
        for (int w = 0; w < kWarps; ++w) below += s.warp_sum[w];
      }
      if (warp == 0) {
        put32_lanes(&s.cand_n[rank], s.sent);
        put32_lanes(&s.own_n[rank], s.n);
        put32_lanes(&s.key_min[rank], s.kmin);
        put32_lanes(&s.key_max[rank], s.kmax);
      }
      sync_all();
      if (const uint32_t c = few ? candidates() : 0u) {
        found_n = c;
        found_k = !by_mass;
        return;
      }
      uint32_t found = 0, most = 0;
      key_lo = 0xFFFFFFFFu;
      key_hi = 0;
      for (int r = 0; r < cs; ++r) {
        found += s.own_n[r];
        most = max(most, s.own_n[r]);
        key_lo = min(key_lo, s.key_min[r]);
        key_hi = max(key_hi, s.key_max[r]);
      }
      if (found <= kList && most <= kOwn) {  // every CTA ranks its share of them (all in each: 256 x 131072 210 us, so 190)
        for (uint32_t i = tid; i < found; i += kThreads) {
          int r = 0;
          uint32_t j = i;
          while (j >= s.own_n[r]) j -= s.own_n[r++];
          const u64 t = ld_cluster_u64(mapa_shared(smem_u32(&s.own[j]), r));
          s.list[i] = t;
          if (by_mass) s.weight[i] = weight(dist(float_of_key(static_cast<uint32_t>(t >> 32))));
        }
        __syncthreads();
        for (uint32_t i = rank * kWarps + warp; i < found; i += cs * kWarps) {  // a warp per token: what comes before it
          const u64 t = s.list[i];
          u64 before = 0;
          if (by_mass) {
            for (uint32_t j = lane; j < found; j += 32) before += s.list[j] > t ? s.weight[j] : 0u;
            before = warp_add(before);
          } else {
            uint32_t c = 0;
            for (uint32_t j = lane; j < found; j += 32) c += s.list[j] > t ? 1u : 0u;
            before = __reduce_add_sync(0xFFFFFFFFu, c);
          }
          if (before < need && need <= before + (by_mass ? s.weight[i] : 1u)) put64_lanes(&s.cut, t);
        }
        sync_all();
        const u64 last = s.cut;
        cut_x = float_of_key(static_cast<uint32_t>(last >> 32));
        cut_i = static_cast<int>(~static_cast<uint32_t>(last));
        if (by_mass) {
          u64 sum = 0;
          for (uint32_t j = lane; j < s.own_n[rank]; j += 32)
            if (s.own[j] >= last) sum += weight(dist(float_of_key(static_cast<uint32_t>(s.own[j] >> 32))));
          cta_mass = below + warp_add(sum);
          known = true;
        }
        return;
      }
      if (key_lo == key_hi) {  // equal logits: so many of them, by index
        const float v = float_of_key(key_lo);
        if (by_mass) {
          const uint32_t w = weight(dist(v));
          need = (need + w - 1) / w;
        }
        auto same = [&](float u, int i) { return u == v && keeps(u, i); };
        uint32_t m = 0;
        each([&](float u, int i) { m += same(u, i) ? 1u : 0u; });
        m = __reduce_add_sync(0xFFFFFFFFu, m);
        __syncthreads();
        if (lane == 0) s.red[warp] = m;
        __syncthreads();
        u64 first = 0;
        for (int w = 0; w < warp; ++w) first += s.red[w];
        for (int r = 0; r < rank; ++r) first += s.own_n[r];
        if (first < need && need <= first + m) {  // (the warp alike)
          for (int st = 0; st < steps && first < need; ++st) {
            uint32_t c = 0;
            four(st, [&](float u, int i) { c += same(u, i) ? 1u : 0u; });
            const u64 to = first + warp_scan(c);
            if (to - c < need && need <= to) {
              u64 at = to - c;
              four(st, [&](float u, int i) {
                if (same(u, i) && ++at == need) {
                  put64(&s.cut, static_cast<uint32_t>(i));
                }
              });
            }
            first = __shfl_sync(0xFFFFFFFFu, to, 31);
          }
        }
        sync_all();
        cut_x = v;
        cut_i = static_cast<int>(s.cut);
        return;
      }
      const int bits = 32 - __clz(key_hi - key_lo);
      shift = max(0, bits - 11);
      ++level;
    }
  };

  if (by_k) shorten(std::false_type{}, static_cast<u64>(top_k), 0.0f);
  // (a top-k that cuts has set cut_x; beside one that does not, the other cuts are as without)
  if (found_n == 0 && cut_x == -INFINITY && min_p > 0.0f && d_max <= kNear) {
    __syncthreads();
    if (tid == 0) s.sent = 0;
    is_empty = false;
    __syncthreads();
    u64 all = 0;
    const bool none = !by_p && !__any_sync(0xFFFFFFFFu, dist(own_mx) <= d_max);
#pragma unroll 1
    for (int st = none ? steps : 0; st < steps; ++st) {
      const float4 v4 = mine4[st * 32 + lane];
      const float v[4] = {v4.x, v4.y, v4.z, v4.w};
      bool in[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float d = dist(v[j]);
        in[j] = d <= d_max;
        if (by_p) all += weight(d);
      }
      send(v, i0 + st * 128, in);
    }
    if (by_p) all = sum_cta(all);
    else __syncthreads();
    if (warp == 0) {
      put32_lanes(&s.cand_n[rank], s.sent);
      put64_lanes(&s.mass[rank], all);
    }
    sync_all();
    const uint32_t found = candidates();
    if (found > 0) {
      found_n = found;
      if (tid == 0) {
        all = 0;
        for (int r = 0; r < cs; ++r) all += s.mass[r];
        s.total = all;
      }
    } else {
      sync_all();  // (the exchanged values have been read)
    }
  }
  if (found_n == 0 && by_p) shorten(std::true_type{}, 0, top_p);
  if (found_n > 0) {
    if (rank == 0) finish(found_n, found_k);
    return;
  }

  auto kept = [&](float v, int i) -> uint32_t {  // the kept weight
    if (v < cut_x) return 0u;
    const float d = dist(v);
    if (!(d <= d_max) || !keeps(v, i)) return 0u;
    const float e = expf(-d);
    return e < min_p ? 0u : __float2uint_rn(e * 2147483648.0f);
  };
  u64 mine = 0;  // of the warp
  auto add_warps = [&]() {
    u64 sum = 0;
    if (cut_x == -INFINITY && min_p == 0.0f) each([&](float v, int) { sum += weight(dist(v)); });
    else each([&](float v, int i) { sum += kept(v, i); });
    mine = warp_add(sum);
    __syncthreads();  // (the sums of a scan before have been read)
    if (lane == 0) s.warp_sum[warp] = mine;
    __syncthreads();
  };
  known = known && min_p == 0.0f;
  if (!known) {
    add_warps();
    cta_mass = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) cta_mass += s.warp_sum[w];
  }
  if (warp == 0) put64_lanes(&s.mass[rank], cta_mass);
  sync_all();
  if (tid == 0) {  // (64-bit floating point is slow: once)
    u64 total = 0;
    for (int r = 0; r < cs; ++r) total += s.mass[r];
    const double want = floor(static_cast<double>(__uint_as_float(s.param[4])) * static_cast<double>(total));
    const u64 r = want > 0.0 ? static_cast<u64>(fmin(want, 9.0e15)) : 0ull;
    s.draw = min(r, total - 1);
    s.total = total;
  }
  __syncthreads();
  const u64 r = s.draw, total = s.total;
  u64 at = 0;
  for (int k = 0; k < rank; ++k) at += s.mass[k];
  if (r < at || r >= at + s.mass[rank]) return;  // another CTA's
  if (known) add_warps();
  for (int w = 0; w < warp; ++w) at += s.warp_sum[w];
  if (at <= r && r < at + mine) {  // (the warp alike)
    // A lane adds up 4 steps consecutive tokens, a scan finds the lane of the
    // drawn number; then its tokens, 32 at a time, one per lane.
    const float* w_x = reinterpret_cast<const float*>(mine4);
    const int t0 = w0 - skip;
    u64 c = 0;
    for (int j = 0; j < steps; ++j) {
      const float4 v = mine4[lane * steps + j];
      const int i = t0 + (lane * steps + j) * 4;
      c += static_cast<u64>(kept(v.x, i)) + kept(v.y, i + 1) + kept(v.z, i + 2) + kept(v.w, i + 3);
    }
    const u64 to = at + warp_scan(c);
    const int owner = __ffs(__ballot_sync(0xFFFFFFFFu, r < to)) - 1;
    at = __shfl_sync(0xFFFFFFFFu, to - c, owner);
    for (int j = 0; j < steps * 4 && at <= r; j += 32) {
      const int e = owner * steps * 4 + j + lane;
      const float v = j + lane < steps * 4 ? w_x[e] : -INFINITY;
      const u64 w = kept(v, t0 + e);
      const u64 upto = at + warp_scan(w);
      if (upto - w <= r && r < upto) {
        a.token[n] = t0 + e;
        if (a.logprob)
          a.logprob[n] = -dist(v) - logf(static_cast<float>(static_cast<double>(total) * 4.656612873077393e-10));
      }
      at = __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
  }
}

// The largest slice a CTA holds: P4Q_MAX_VOCAB over a full cluster, with a row's
// misalignment, in whole steps of its warps.
constexpr int kMaxSteps = 18;

template <int kType>
cudaError_t launch_type(const SampleArgs& a, cudaStream_t stream) {
  constexpr int kSize = kType == 2 ? 4 : 2;
  constexpr int kStep = kType == 2 ? 1 : 2;  // a warp's 16-byte loads are one or two steps of 128 elements
  // the row's elements from the 16-byte boundary before it, at the worst alignment that the rows have
  const bool aligned = (reinterpret_cast<uintptr_t>(a.logits) & 15u) == 0 && (a.ld * kSize) % 16 == 0;
  const int elements = a.vocab + (aligned ? 0 : 16 / kSize - 1);
  auto steps_of = [&](int cs) {
    const int unit = 128 * kStep * kWarps * cs;
    return (elements + unit - 1) / unit * kStep;
  };
  // CTAs per row: so that every SM has one, eight only while no SM gets two, and no
  // slice is longer than 16384 (if a larger cluster can be had). Eight and four at 32 x
  // 32000 fp16: plain 6.9, 6.8, top-k 14.3, 8.3, top-p 17.8, 17.4; at 16 x 32000 6.6, 6.7,
  // 9.3, 8.3, 16.5, 17.3; at 8 x 65536 fp32 6.8, 8.7, 8.7, 9.0, 17.2, 23.0. Plain draws / top-p with clusters of 1, 2, 4, 8,
  // us: 1 x 32000 fp16 10.9, 7.5, 5.6, 5.2 / 27.6, 21.4, 15.0, 13.8; 64 x 32000
  // 14.1, 9.5, 8.2, 11.9 / 32.0, 21.6, 18.9, 30.0; 256 x 32000 bf16 25.0, 20.3,
  // 24.7, 39.0 / 60.8, 49.1, 62.2, 106; 256 x 131072 fp32 (4 and 8) 76.0, 64.8 /
  // 218, 193.
  int cs = 1;
  while (cs < kMaxCluster && ((2 * cs < kMaxCluster ? a.rows * cs < num_sms() : a.rows * 2 * cs <= num_sms()) || steps_of(cs) > 8))
    cs *= 2;
  const int steps = steps_of(cs);
  if (steps > kMaxSteps) return cudaErrorInvalidValue;
  static SmemLimit limit;
  const cudaError_t e = limit.allow(sample_kernel<kType>, kMaxSteps * kWarps * 512);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows) * static_cast<unsigned>(cs));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(steps) * kWarps * 512;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(cs);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cs > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<kType>, a, steps);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, cudaStream_t stream) {
  return a.dtype == 2 ? launch_type<2>(a, stream) : a.dtype == 1 ? launch_type<1>(a, stream) : launch_type<0>(a, stream);
}

}  // namespace p4q
