// The draw of one token from each row of logits: temperature, top-k, top-p and
// min-p with a given uniform number.
//
// Weights are integers (2^31 exp(-d) rounded), so that their sums are exact and
// the drawn token depends on no order of summation, hence on no split of the
// row either. The kept tokens are a head of the row in the order "falling logit,
// then rising index"; each cut is the last token of that head.
//
// A cluster of CTAs takes a row; its logits are read once and stay in shared
// memory, a slice of the row in each CTA (in registers, 32 a thread, the values
// that the passes below derive from them spilled).
// A cut is found as follows. A histogram over d in steps of 1 / 92 (counts for
// top-k, weights for top-p) covers every token whose weight is not 0 (2^31 e^-d
// rounds to 0 past d = 22.2; those come last and are never drawn, so they take
// no part). The CTAs add up a slice of the bins each, scan it, and the bin in
// which the wanted sum is reached follows. Its tokens, mostly a few, go to
// one list and are ranked. Bins of more tokens than the list holds are divided
// again by the logits' ordered bit patterns, at most three times (11 of 32 bits
// each); a bin of equal logits is cut by index. Shared-memory atomics are what
// a histogram costs, so tokens that the cut cannot reach stay out of it: for
// top-k those below the k-th of the threads' own maxima (a CTA alone has k tokens
// above it), for top-p those whose weights, all of them together, are less than
// what may be cut off.
// The draw: kept weights per warp (a warp's tokens are consecutive), their prefix
// over the cluster, and the one warp that contains the drawn number walks
// its tokens.
#include <climits>
#include <cuda_runtime.h>

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
constexpr int kList = 512;

struct Shared {
  uint32_t lo[kBins], hi[kBins];  // counts, or the weights' low and high 16 bits
  uint32_t lkey[kList], lidx[kList], lw[kList];
  u64 warp_sum[kWarps];
  // written by the other CTAs of the cluster
  u64 slice_total[kMaxCluster], mass[kMaxCluster], sum[kMaxCluster], ties[kMaxCluster];
  uint32_t max_key[kMaxCluster], first_max[kMaxCluster];
  u64 need;
  uint32_t bin, cut_key, cut_idx;
  uint32_t list_n, key_min, key_max;  // (of the cluster's first CTA)
  uint32_t red[kWarps];
  int last_bin;  // (of this CTA)
};

__device__ __forceinline__ float float_of_key(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t add_cluster_u32(uint32_t a, uint32_t v) {
  uint32_t old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(a), "r"(v) : "memory");
  return old;
}

__device__ __forceinline__ void min_cluster_u32(uint32_t a, uint32_t v) {
  asm volatile("red.shared::cluster.min.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}

__device__ __forceinline__ void max_cluster_u32(uint32_t a, uint32_t v) {
  asm volatile("red.shared::cluster.max.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
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
  auto put32 = [&](uint32_t* p, uint32_t v) {  // the variable in every CTA of the cluster
    for (int r = 0; r < cs; ++r) st_shared_cluster_u32(mapa_shared(smem_u32(p), r), v);
  };
  auto put64 = [&](u64* p, u64 v) {
    put32(reinterpret_cast<uint32_t*>(p), static_cast<uint32_t>(v));
    put32(reinterpret_cast<uint32_t*>(p) + 1, static_cast<uint32_t>(v >> 32));
  };
  auto at_first = [&](uint32_t* p) { return mapa_shared(smem_u32(p), 0); };

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
  float4* const mine4 = xs + warp * steps * 32;
  auto clean = [](float v) { return v != v ? -INFINITY : v + 0.0f; };  // NaN counts as -inf, -0 as +0
  float mx = -INFINITY;
  if (kType == 2) {
#pragma unroll 4
    for (int st = 0; st < steps; ++st) {
      const int e = w0 + (st * 32 + lane) * 4;
      float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      const float* p = reinterpret_cast<const float*>(row) + e;
      if (e >= skip && e + 4 <= end) {
        v = *reinterpret_cast<const float4*>(p);
      } else {
        if (e >= skip && e < end) v.x = p[0];
        if (e + 1 >= skip && e + 1 < end) v.y = p[1];
        if (e + 2 >= skip && e + 2 < end) v.z = p[2];
        if (e + 3 >= skip && e + 3 < end) v.w = p[3];
      }
      v = make_float4(clean(v.x), clean(v.y), clean(v.z), clean(v.w));
      mine4[st * 32 + lane] = v;
      mx = fmaxf(fmaxf(fmaxf(mx, v.x), fmaxf(v.y, v.z)), v.w);
    }
  } else {
    // 8 elements per lane and 16-byte piece (steps is even)
#pragma unroll 4
    for (int st = 0; st < steps / 2; ++st) {
      const int e = w0 + (st * 32 + lane) * 8;
      const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + e;
      uint32_t raw[4];
      if (e >= skip && e + 8 <= end) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        raw[0] = v.x;
        raw[1] = v.y;
        raw[2] = v.z;
        raw[3] = v.w;
      } else {
        constexpr uint32_t kNone = kType == 1 ? 0xFF80u : 0xFC00u;  // -inf
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t l = e + 2 * j >= skip && e + 2 * j < end ? p[2 * j] : kNone;
          const uint32_t h = e + 2 * j + 1 >= skip && e + 2 * j + 1 < end ? p[2 * j + 1] : kNone;
          raw[j] = l | (h << 16);
        }
      }
      float f[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = unpack2<kType == 1>(raw[j]);
        f[2 * j] = clean(v.x);
        f[2 * j + 1] = clean(v.y);
        mx = fmaxf(mx, fmaxf(f[2 * j], f[2 * j + 1]));
      }
      mine4[(st * 32 + lane) * 2] = make_float4(f[0], f[1], f[2], f[3]);
      mine4[(st * 32 + lane) * 2 + 1] = make_float4(f[4], f[5], f[6], f[7]);
    }
  }
  const float own_max = mx;
  __syncwarp();
  // f(logit, token) for this lane's four tokens of a step
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
#pragma unroll 2
    for (int st = 0; st < steps; ++st) four(st, f);
  };

  // the row's largest logit
  {
    const uint32_t k = __reduce_max_sync(0xFFFFFFFFu, float_order_key(mx));
    if (lane == 0) s.red[warp] = k;
    if (tid == 0) {
      s.list_n = 0;
      s.key_min = 0xFFFFFFFFu;
      s.key_max = 0;
    }
    __syncthreads();
    if (warp == 0) {
      const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, s.red[lane & (kWarps - 1)]);
      if (lane == 0) put32(&s.max_key[rank], all);
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
  const float temp = a.temperature ? a.temperature[n] : 1.0f;
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
      st_shared_cluster_u32(at_first(&s.first_max[rank]), first);
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
  auto d_bin = [&](float d, int* bin) {  // false: past the bins
    const float f = fmaf(d, kBinScale, 8388608.0f);  // d in bins, rounded, behind 2^23
    *bin = __float_as_int(f) & 0x7FFFFF;
    return f < 8388608.0f + kBins;
  };
  float cut_x = -INFINITY;  // the last kept token
  int cut_i = INT_MAX;
  auto keeps = [&](float v, int i) { return v > cut_x || (v == cut_x && i <= cut_i); };
  // A sum over the cluster's threads; *before: that of the warps before this one.
  auto sum_all = [&](u64 v, u64* slots, u64* before) -> u64 {
    v = warp_add(v);
    __syncthreads();  // (the sums of a scan before have been read)
    if (lane == 0) s.warp_sum[warp] = v;
    __syncthreads();
    u64 cta = 0, at = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) at += s.warp_sum[w];
      cta += s.warp_sum[w];
    }
    if (tid == 0) put64(&slots[rank], cta);
    sync_all();
    u64 total = 0;
    for (int r = 0; r < cs; ++r) {
      if (r < rank) at += slots[r];
      total += slots[r];
    }
    *before = at;
    return total;
  };

  // Shortens the kept head: to `need` tokens (by_mass false), or to the first
  // tokens whose weights reach ceil(share * the kept weights' sum).
  auto shorten = [&](const bool by_mass, u64 need, float share) {
    const bool all_kept = cut_x == -INFINITY;
    auto reach = [&](u64 total) -> u64 {
      const double want = ceil(static_cast<double>(share) * static_cast<double>(total));
      return want < 1.0 ? 1ull : static_cast<u64>(want);
    };
    int last_bin = kBins - 1;  // tokens of later bins are past the cut
    if (by_mass && all_kept) {
      u64 sum = 0, before;
      each([&](float v, int i) { sum += weight(dist(v)); });
      sum = sum_all(sum, s.sum, &before);
      need = reach(sum);
      // Tokens of weight <= (sum - need) / V have no more than sum - need together. Bin b + 1 begins half a
      // bin behind b's middle, and a weight is off by half a unit: one unit and one bin less.
      const float spare = static_cast<float>((sum - need) / static_cast<unsigned int>(V));
      if (spare > 2.0f) last_bin = min(last_bin, static_cast<int>((21.487563f - logf(spare - 1.0f)) * kBinScale) + 2);
    }
    for (int i = tid; i < kBins; i += kThreads) {
      s.lo[i] = 0;
      s.hi[i] = 0;
    }
    __syncthreads();
    if (!by_mass && need <= kThreads) {
      // the bin of the need-th of the threads' largest logits (in the array that counts leave free)
      int bin;
      if (d_bin(dist(own_max), &bin)) atomicAdd(&s.hi[bin], 1u);
      if (tid == 0) s.last_bin = kBins - 1;
      __syncthreads();
      constexpr int kPer = kBins / kThreads;
      uint32_t c[kPer], own = 0;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        c[j] = s.hi[tid * kPer + j];
        own += c[j];
      }
      uint32_t upto = own;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += v;
      }
      if (lane == 31) s.red[warp] = upto;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        if (w < warp) upto += s.red[w];
      if (own > 0 && upto >= need && upto - own < need) {
        uint32_t at = upto - own;
        int j = 0;
        while ((at += c[j]) < need) ++j;
        s.last_bin = tid * kPer + j;
      }
      __syncthreads();
      last_bin = s.last_bin;
    }
    uint32_t key_lo = 0, key_hi = 0;
    int shift = 0;
    for (int level = 0;; ++level) {
      // the bin of a token (falling logits have rising bins), or -1
      auto bin_of = [&](float v, int i) -> int {
        if (level == 0) {
          int bin;
          return d_bin(dist(v), &bin) && bin <= last_bin && keeps(v, i) ? bin : -1;
        }
        const uint32_t k = float_order_key(v);
        return k >= key_lo && k <= key_hi && keeps(v, i) ? static_cast<int>((key_hi - k) >> shift) : -1;
      };
      if (level > 0) {
        for (int i = tid; i < kBins; i += kThreads) {
          s.lo[i] = 0;
          s.hi[i] = 0;
        }
        __syncthreads();
      }
      each([&](float v, int i) {
        const int bin = bin_of(v, i);
        if (bin >= 0) {
          if (by_mass) {
            const uint32_t w = weight(dist(v));
            atomicAdd(&s.lo[bin], w & 0xFFFFu);
            if (w >> 16) atomicAdd(&s.hi[bin], w >> 16);
          } else {
            atomicAdd(&s.lo[bin], 1u);
          }
        }
      });
      sync_all();
      if (rank == 0 && tid == 0) {
        s.list_n = 0;
        s.key_min = 0xFFFFFFFFu;
        s.key_max = 0;
      }
      // this CTA's slice of the bins over the cluster, `per` bins per thread
      const int slice = kBins / cs, per = max(1, slice / kThreads);
      u64 bins[kBins / kThreads], own = 0;
#pragma unroll
      for (int j = 0; j < kBins / kThreads; ++j) {
        bins[j] = 0;
        if (j < per && tid * per < slice) {
          const int bin = rank * slice + tid * per + j;
#pragma unroll
          for (int r = 0; r < kMaxCluster; ++r)
            if (r < cs) {
              bins[j] += ld_cluster_u32(mapa_shared(smem_u32(&s.lo[bin]), r));
              if (by_mass) bins[j] += static_cast<u64>(ld_cluster_u32(mapa_shared(smem_u32(&s.hi[bin]), r))) << 16;
            }
        }
        own += bins[j];
      }
      u64 upto = warp_scan(own);
      if (lane == 31) s.warp_sum[warp] = upto;
      __syncthreads();
      u64 all = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) upto += s.warp_sum[w];
        all += s.warp_sum[w];
      }
      if (tid == 0) put64(&s.slice_total[rank], all);
      sync_all();
      u64 total = 0;
      for (int r = 0; r < cs; ++r) {
        if (r < rank) upto += s.slice_total[r];
        total += s.slice_total[r];
      }
      if (level == 0) {
        if (by_mass && !all_kept) need = reach(total);
        if (total < need) return;  // fewer tokens than `need` may be drawn at all
      }
      if (own > 0 && upto - own < need && need <= upto) {
        u64 at = upto - own;
        int j = 0;
        while (j + 1 < per && at + bins[j] < need) at += bins[j++];
        put32(&s.bin, static_cast<uint32_t>(rank * slice + tid * per + j));
        put64(&s.need, need - at);
      }
      sync_all();
      const int bin = static_cast<int>(s.bin);
      need = s.need;
      // its tokens into the first CTA's list
      uint32_t c = 0, kmin = 0xFFFFFFFFu, kmax = 0;
      each([&](float v, int i) {
        if (bin_of(v, i) == bin) {
          const uint32_t k = float_order_key(v);
          ++c;
          kmin = min(kmin, k);
          kmax = max(kmax, k);
        }
      });
      const uint32_t in_warp = __reduce_add_sync(0xFFFFFFFFu, c);
      if (in_warp > 0) {
        kmin = __reduce_min_sync(0xFFFFFFFFu, kmin);
        kmax = __reduce_max_sync(0xFFFFFFFFu, kmax);
        const uint32_t before = static_cast<uint32_t>(warp_scan(c)) - c;
        uint32_t at = 0;
        if (lane == 0) {
          at = add_cluster_u32(at_first(&s.list_n), in_warp);
          min_cluster_u32(at_first(&s.key_min), kmin);
          max_cluster_u32(at_first(&s.key_max), kmax);
        }
        at = __shfl_sync(0xFFFFFFFFu, at, 0) + before;
        if (c > 0 && at < kList) {
          each([&](float v, int i) {
            if (bin_of(v, i) == bin && at < kList) {
              st_shared_cluster_u32(at_first(&s.lkey[at]), float_order_key(v));
              st_shared_cluster_u32(at_first(&s.lidx[at]), static_cast<uint32_t>(i));
              if (by_mass) st_shared_cluster_u32(at_first(&s.lw[at]), weight(dist(v)));
              ++at;
            }
          });
        }
      }
      sync_all();
      const uint32_t found = ld_cluster_u32(at_first(&s.list_n));
      key_lo = ld_cluster_u32(at_first(&s.key_min));
      key_hi = ld_cluster_u32(at_first(&s.key_max));
      if (found <= kList) {  // every CTA ranks them for itself
        uint32_t k = 0, i = 0, w = 1;
        if (tid < static_cast<int>(found)) {
          k = ld_cluster_u32(at_first(&s.lkey[tid]));
          i = ld_cluster_u32(at_first(&s.lidx[tid]));
          if (by_mass) w = ld_cluster_u32(at_first(&s.lw[tid]));
          if (rank > 0) {
            s.lkey[tid] = k;
            s.lidx[tid] = i;
            if (by_mass) s.lw[tid] = w;
          }
        }
        __syncthreads();
        if (tid < static_cast<int>(found)) {
          u64 before = 0;
          for (uint32_t j = 0; j < found; ++j) {
            const uint32_t kj = s.lkey[j];
            if (kj > k || (kj == k && s.lidx[j] < i)) before += by_mass ? s.lw[j] : 1u;
          }
          if (before < need && need <= before + w) {
            s.cut_key = k;
            s.cut_idx = i;
          }
        }
        __syncthreads();
        break;
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
        if (lane == 0) s.red[warp] = m;
        __syncthreads();
        u64 cta = 0, first = 0;
        for (int w = 0; w < kWarps; ++w) {
          if (w < warp) first += s.red[w];
          cta += s.red[w];
        }
        if (tid == 0) put64(&s.ties[rank], cta);
        sync_all();
        for (int r = 0; r < rank; ++r) first += s.ties[r];
        if (first < need && need <= first + m) {  // (the warp alike)
          for (int st = 0; st < steps && first < need; ++st) {
            uint32_t mine = 0;
            four(st, [&](float u, int i) { mine += same(u, i) ? 1u : 0u; });
            const u64 to = first + warp_scan(mine);
            if (to - mine < need && need <= to) {
              u64 at = to - mine;
              four(st, [&](float u, int i) {
                if (same(u, i) && ++at == need) {
                  put32(&s.cut_key, key_lo);
                  put32(&s.cut_idx, static_cast<uint32_t>(i));
                }
              });
            }
            first = __shfl_sync(0xFFFFFFFFu, to, 31);
          }
        }
        sync_all();
        break;
      }
      const int bits = 32 - __clz(key_hi - key_lo);
      shift = max(0, bits - 11);
    }
    cut_x = float_of_key(s.cut_key);
    cut_i = static_cast<int>(s.cut_idx);
  };

  const int top_k = a.top_k ? a.top_k[n] : 0;
  if (top_k > 0 && top_k < V) shorten(false, static_cast<u64>(top_k), 0.0f);
  const float top_p = a.top_p ? a.top_p[n] : 1.0f;
  if (top_p < 1.0f) shorten(true, 0, top_p);

  const float min_p = a.min_p && a.min_p[n] > 0.0f ? fminf(a.min_p[n], 1.0f) : 0.0f;
  // past d_max exp(-d) < min_p for certain (weights are 0 past 22.2)
  const float d_max = fminf(min_p > 0.0f ? 1e-5f - 1.000001f * logf(min_p) : 23.0f, 23.0f);
  auto kept = [&](float v, int i) -> uint32_t {  // the kept weight
    const float d = dist(v);
    if (!(d <= d_max) || !keeps(v, i)) return 0u;
    const float e = expf(-d);
    return e < min_p ? 0u : __float2uint_rn(e * 2147483648.0f);
  };
  u64 mine = 0, at;
  each([&](float v, int i) { mine += kept(v, i); });
  mine = warp_add(mine);
  const u64 total = sum_all(lane == 0 ? mine : 0ull, s.mass, &at);
  const double want = floor(static_cast<double>(a.u[n]) * static_cast<double>(total));
  u64 r = want > 0.0 ? static_cast<u64>(fmin(want, 9.0e15)) : 0ull;
  if (r > total - 1) r = total - 1;
  if (at <= r && r < at + mine) {  // (the warp alike)
    for (int st = 0; st < steps && at <= r; ++st) {
      u64 c = 0;
      four(st, [&](float v, int i) { c += kept(v, i); });
      const u64 to = at + warp_scan(c);
      if (to - c <= r && r < to) {
        u64 w = to - c;
        bool done = false;
        four(st, [&](float v, int i) {
          w += kept(v, i);
          if (!done && w > r) {
            done = true;
            a.token[n] = i;
            if (a.logprob)
              a.logprob[n] = -dist(v) - logf(static_cast<float>(static_cast<double>(total) * 4.656612873077393e-10));
          }
        });
      }
      at = __shfl_sync(0xFFFFFFFFu, to, 31);
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
  int cs = 1;
  while (cs < kMaxCluster && (a.rows * cs < num_sms() || steps_of(cs) > 8)) cs *= 2;
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
