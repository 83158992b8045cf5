// Attention of one new token per sequence for groups of sequences that share a prefix: the
// prefix's keys and values are read once per group instead of once per sequence.
//
// Two kernels. prefix_kernel takes the prefixes: with n sequences of G query heads per
// key/value head there are n G rows of queries to the same keys, enough for the tensor cores'
// 128-row products (tcgen05 kind::f16, fp32 accumulators in TMEM). The paged attention kernel
// (p4q_paged_kernel.cuh) takes the positions that each sequence has of its own, adds the
// prefix's parts at its end and writes the outputs. It needs nothing of the first before
// that, so it starts beside it, on what the first leaves free of the SMs.
//
// prefix_kernel: units and ranges as p4q_paged_prefix.cuh says. Nine warps:
//   warps 0-3  queries, keys and values into shared memory with 16-byte asynchronous copies (pages
//              may be of any size and order, and positions past the prefix or of a page outside the
//              cache have to be zeros: 0 weight times an infinite value is NaN), in the 128-byte
//              swizzle that the products read; two stages each of keys and values;
//   warps 4-7  one thread per row (its TMEM lane): scores' maximum, p = 2^(s - reference),
//              their sum, p as two fp16 or three bf16 values over the scores in TMEM; the
//              reference moves, and O with it, only when a score exceeds it by 2^4 (bf16 2^8);
//   warp 8     issues the products: S = Q K^T of the next chunk, then O += P V of this one, with
//              P from TMEM and V in place as an MN-major operand.
// p goes into the product in parts for the reasons that p4q_paged_rows.cuh gives, by the same
// rules. Every wait is bounded; a time-out sets the device error word.
#include <cuda_runtime.h>

#include <algorithm>

#include "p4q_paged_kernel.cuh"
#include "p4q_paged_rows.cuh"

namespace p4q {
namespace {

__device__ unsigned int g_prefix_wait_err;

constexpr int kProducers = 4, kSoftmax = 4;          // warps
constexpr int kPrefixThreads = 32 * (kProducers + kSoftmax + 1);
constexpr int kMaxPrefixGrid = 160;
constexpr int kTileBytes = 16384;                    // 128 rows of 128 bytes
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 128, kSCols = 192;        // O: columns 0 .. 127; two S buffers, with room for P's third part
constexpr int kMetas = 4;                            // of chunks' valid positions, see the producers

struct Bars {
  uint64_t q_full, q_empty, k_full[2], k_empty[2], v_full[2], v_empty[2], meta_full[kMetas];
  uint64_t s_full[2], p_ready[2], pv_done[2], o_free, mma_done;
  unsigned long long first, base, share, total;  // the CTA's range and the start of its first group
  int group;
  uint32_t valid[kMetas][kProducers];
  uint32_t tmem_slot;
  int abort_flag;
};

template <int kDh>
constexpr int smem_bytes() {
  return (kDh / 64) * kTileBytes * 5 + static_cast<int>(sizeof(Bars)) + 1024;
}

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool full) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(full ? 16 : 0) : "memory");
}

// Arrives on `bar` once this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
      "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
      "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// kind::f16 with fp16 or bf16 A and B (K-major; bit 16 set: B MN-major) and an fp32 accumulator, M x N.
template <bool kBf16>
constexpr uint32_t idesc16(int M, int N) {
  return (1u << 4) | (kBf16 ? (1u << 7) | (1u << 10) : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}

// A and B from shared memory.
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// A from TMEM (lanes = rows, two values of K per column), B from shared memory.
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// MN-major operand in 128-byte swizzled atoms: 8 rows of K x 64 values along MN per 1024 bytes,
// atoms every 1024 bytes along K and every `mn_stride` bytes along MN.
__device__ __forceinline__ uint64_t mn_major_desc(uint32_t saddr, uint32_t mn_stride) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | static_cast<uint64_t>(mn_stride >> 4) << 16 |
         static_cast<uint64_t>(1024 >> 4) << 32 | static_cast<uint64_t>(1) << 46 | static_cast<uint64_t>(2) << 61;
}

// A CTA's range, unit by unit: chunks c0 .. c1 - 1 of tile `tile` of key/value head hk of the
// group gr. Every role walks it by itself.
struct Walk {
  unsigned long long x, end, base;
  int g;
  Group gr;
  int hk, tile, c0, c1;
  __device__ Walk(const PrefixArgs& a, const Bars& br) : x(br.first), base(br.base), g(br.group) {
    end = min(br.total, x + br.share);
    if (x < end) {
      gr = load_group(a, g);
      find(a);
    }
  }
  __device__ bool more() const { return x < end; }
  __device__ void find(const PrefixArgs& a) {
    while (x >= base + group_chunks(a, gr)) {  // (x < total: such a group comes)
      base += group_chunks(a, gr);
      gr = load_group(a, ++g);
    }
    const unsigned int at = static_cast<unsigned int>((x - base) / static_cast<unsigned int>(gr.chunks));
    c0 = static_cast<int>(x - base - static_cast<unsigned long long>(at) * gr.chunks);
    c1 = static_cast<int>(min(static_cast<unsigned long long>(gr.chunks), c0 + (end - x)));
    hk = static_cast<int>(at) / gr.tiles;
    tile = static_cast<int>(at) - hk * gr.tiles;
  }
  __device__ void next(const PrefixArgs& a) {
    x += c1 - c0;
    if (x < end) find(a);
  }
};

template <bool kBf16, int kDh>
__global__ void __launch_bounds__(kPrefixThreads, 1) prefix_kernel(const PrefixArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  constexpr int kHalves = kDh / 64;                 // 128-byte halves of a row
  constexpr int kOperand = kHalves * kTileBytes;
  constexpr int kOffK = kOperand, kOffV = 3 * kOperand, kOffBars = 5 * kOperand;
  constexpr int kPw = kParts<kBf16>;
  Bars& br = *reinterpret_cast<Bars*>(smem + kOffBars);
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  volatile int* const abort_flag = &br.abort_flag;
  const PagedCache& c = a.kv;
  const int G = a.H / c.Hkv;

  if (t == 0) {
    mbar_init(&br.q_full, 32 * kProducers);
    mbar_init(&br.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&br.k_full[i], 32 * kProducers);
      mbar_init(&br.k_empty[i], 1);
      mbar_init(&br.v_full[i], 32 * kProducers);
      mbar_init(&br.v_empty[i], 1);
      mbar_init(&br.s_full[i], 1);
      mbar_init(&br.p_ready[i], kSoftmax);
      mbar_init(&br.pv_done[i], 1);
    }
    for (int i = 0; i < kMetas; ++i) mbar_init(&br.meta_full[i], kProducers);
    mbar_init(&br.o_free, kSoftmax);
    mbar_init(&br.mma_done, 1);
    br.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 8) {
    tmem_alloc(&br.tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_launch_dependents();
  if (warp == 0) {
    // the chunks before each group, their sum, and the group that the CTA's range begins in
    unsigned long long total = 0;
    for (int pass = 0; pass < 2; ++pass) {
      const unsigned long long share = prefix_share(total, a.grid), first = blockIdx.x * share;
      unsigned long long upto = 0;
      for (int g0 = 0; g0 < a.groups; g0 += 32) {
        const int g = g0 + lane;
        unsigned long long n = 0;
        if (g < a.groups) {
          n = group_chunks(a, load_group(a, g));
          if (pass == 0 && blockIdx.x == 0 &&
              (a.group_start[g] < 0 || a.group_start[g + 1] < a.group_start[g] || a.group_start[g + 1] > c.seqs ||
               a.prefix_lens[g] > paged_room(c)))
            atomicOr(&g_paged_err, kErrIndex);
        }
        unsigned long long s = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const unsigned long long v = __shfl_up_sync(0xFFFFFFFFu, s, d);
          if (lane >= d) s += v;
        }
        const unsigned long long before = upto + s - n;
        if (pass == 1) {
          if (blockIdx.x == 0 && g < a.groups) a.base[g] = before;
          if (g < a.groups && first >= before && first < before + n) {
            br.group = g;
            br.base = before;
          }
        }
        upto += __shfl_sync(0xFFFFFFFFu, s, 31);
      }
      if (pass == 0) {
        total = upto;
      } else if (lane == 0) {
        if (blockIdx.x == 0) a.base[a.groups] = total;
        br.first = first;
        br.share = share;
        br.total = total;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = br.tmem_slot;

  if (warp < kProducers) {
    // ---------------------------------------------------------------- queries, keys, values
    constexpr int kPieces = 8 * kHalves;      // 16-byte pieces of a row
    constexpr int kRowsAtOnce = 32 / kPieces;  // of a warp
    const int piece = lane & (kPieces - 1), sub = lane / kPieces;
    bool ok = true;
    // the warp's 32 rows of a tile, one address per lane; zeros where there is none
    auto copy_rows = [&](uint8_t* tile, const uint16_t* row, const uint16_t* any) {
      const unsigned long long mine = reinterpret_cast<unsigned long long>(row);
#pragma unroll 8
      for (int i = 0; i < 32; i += kRowsAtOnce) {
        const unsigned long long src = __shfl_sync(0xFFFFFFFFu, mine, i + sub);
        const int r = warp * 32 + i + sub;
        const uint32_t dst = smem_u32(tile) + (piece >> 3) * kTileBytes + r * 128 + (((piece & 7) ^ (r & 7)) << 4);
        cp_async16_or_zero(dst, src ? reinterpret_cast<const uint16_t*>(src) + piece * 8 : any, src != 0);
      }
    };
    int j = 0, uq = 0;
    for (Walk w(a, br); w.more() && ok; w.next(a), ++uq) {
      const int32_t* const table = c.table + static_cast<long long>(w.gr.first) * c.table_ld;
      auto page_of = [&](int chunk) -> int {  // of this lane's position of a chunk
        const int p = chunk * kPrefixChunk + warp * 32 + lane;
        return p < w.gr.prefix && chunk < w.c1 ? table[p >> c.page_log2] : -1;
      };
      int page = page_of(w.c0);
      if (uq > 0) ok = mbar_wait_all(&br.q_empty, (uq - 1) & 1, abort_flag, &g_prefix_wait_err);
      if (!ok) break;
      const int idx = w.tile * kPrefixRows + warp * 32 + lane;
      const uint16_t* qrow = nullptr;
      if (idx < w.gr.n * G)
        qrow = a.q + (w.gr.first + idx / G) * a.ldq + static_cast<long long>(w.hk * G + idx % G) * kDh;
      copy_rows(smem, qrow, a.q);
      cp_async_arrive(&br.q_full);
      for (int ch = w.c0; ch < w.c1; ++ch, ++j) {
        const int st = j & 1;
        const int p = ch * kPrefixChunk + warp * 32 + lane;
        const bool valid = p < w.gr.prefix && static_cast<unsigned int>(page) < static_cast<unsigned int>(c.pages);
        const long long off = valid ? page * c.page_stride + (p & ((1 << c.page_log2) - 1)) * c.token_stride + w.hk * c.head_stride : 0;
        page = page_of(ch + 1);
        if (j >= 2) ok = mbar_wait_all(&br.k_empty[st], ((j >> 1) - 1) & 1, abort_flag, &g_prefix_wait_err);
        if (!ok) break;
        // The scores' warps read it after S of this chunk, whose product ran before that of chunk
        // j + kMetas - 2 released the stage that is waited for here; by then they had
        // this chunk's P ready, which the P V before that product waits for.
        const uint32_t bits = __ballot_sync(0xFFFFFFFFu, valid);
        if (lane == 0) {
          br.valid[j & (kMetas - 1)][warp] = bits;
          mbar_arrive(&br.meta_full[j & (kMetas - 1)]);
        }
        copy_rows(smem + kOffK + st * kOperand, valid ? c.k + off : nullptr, c.k);
        cp_async_arrive(&br.k_full[st]);
        if (j >= 2) ok = mbar_wait_all(&br.v_empty[st], ((j >> 1) - 1) & 1, abort_flag, &g_prefix_wait_err);
        if (!ok) break;
        copy_rows(smem + kOffV + st * kOperand, valid ? c.v + off : nullptr, c.v);
        cp_async_arrive(&br.v_full[st]);
      }
    }
    cp_async_commit();
    cp_async_wait<0>();  // nothing of this CTA's copies may be in flight when it exits
  } else if (warp == 8) {
    // ---------------------------------------------------------------- products
    const bool leader = elect_one();
    bool ok = true;
    constexpr uint32_t idS = idesc16<kBf16>(kPrefixRows, kPrefixChunk);
    constexpr uint32_t idO = idesc16<kBf16>(kPrefixRows, kDh) | (1u << 16);  // V MN-major
    const uint64_t q_desc = sw128_kmajor_desc(smem_u32(smem));
    const uint64_t k_desc = sw128_kmajor_desc(smem_u32(smem + kOffK));
    const uint64_t v_desc = mn_major_desc(smem_u32(smem + kOffV), kTileBytes);
    // S = Q K^T of the chunk that s stands at, into buffer js & 1 (which held the P of chunk js - 2,
    // whose P V was issued before: products of one thread run in order).
    Walk s(a, br);
    int js = 0, us = 0, cs = s.more() ? s.c0 : 0;
    auto issue_s = [&]() {
      const int st = js & 1;
      if (cs == s.c0) ok = ok && mbar_wait_all(&br.q_full, us & 1, abort_flag, &g_prefix_wait_err);
      ok = ok && mbar_wait_all(&br.k_full[st], (js >> 1) & 1, abort_flag, &g_prefix_wait_err);
      if (!ok) return;
      fence_proxy_async_smem();  // the copies are seen by the products
      tc_fence_after();
      const uint32_t d = tmem + kColS + kSCols * static_cast<uint32_t>(st);
      const uint64_t b0 = k_desc + static_cast<uint32_t>(st * (kOperand >> 4));
      const bool last = cs + 1 == s.c1;
      if (leader) {
#pragma unroll
        for (int kb = 0; kb < kHalves; ++kb)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_ss(d, q_desc + kb * (kTileBytes >> 4) + 2 * k, b0 + kb * (kTileBytes >> 4) + 2 * k, idS, (kb | k) != 0 ? 1u : 0u);
        mma_commit(&br.s_full[st]);
        mma_commit(&br.k_empty[st]);
        if (last) mma_commit(&br.q_empty);
      }
      ++js;
      if (last) {
        s.next(a);
        ++us;
        cs = s.more() ? s.c0 : 0;
      } else {
        ++cs;
      }
    };
    if (s.more()) issue_s();
    int j = 0, uq = 0;
    for (Walk w(a, br); w.more() && ok; w.next(a), ++uq) {
      for (int ch = w.c0; ch < w.c1 && ok; ++ch, ++j) {
        if (s.more()) issue_s();
        const int st = j & 1;
        ok = ok && mbar_wait_all(&br.p_ready[st], (j >> 1) & 1, abort_flag, &g_prefix_wait_err);
        if (ch == w.c0 && uq > 0) ok = ok && mbar_wait_all(&br.o_free, (uq - 1) & 1, abort_flag, &g_prefix_wait_err);
        ok = ok && mbar_wait_all(&br.v_full[st], (j >> 1) & 1, abort_flag, &g_prefix_wait_err);
        if (!ok) break;
        fence_proxy_async_smem();
        tc_fence_after();
        const uint32_t pa = tmem + kColS + kSCols * static_cast<uint32_t>(st);
        const uint64_t b0 = v_desc + static_cast<uint32_t>(st * (kOperand >> 4));
        if (leader) {
#pragma unroll
          for (int kt = 0; kt < kPrefixChunk / 16; ++kt)  // 16 positions per product: 8 columns of P, 16 rows of V
#pragma unroll
            for (int i = 0; i < kPw; ++i)
              mma_ts(tmem, pa + (i < 2 ? 32u * (kt >> 1) + 16u * i + 8u * (kt & 1) : 128u + 8u * kt), b0 + (2048 >> 4) * kt, idO,
                     (ch > w.c0 || kt > 0 || i > 0) ? 1u : 0u);
          mma_commit(&br.v_empty[st]);
          mma_commit(&br.pv_done[st]);
        }
      }
    }
    if (leader) {  // every product has completed before TMEM is released
      mma_commit(&br.mma_done);
      volatile int never = 0;
      mbar_wait(&br.mma_done, 0, &never, &g_prefix_wait_err);
    }
  } else {
    // ---------------------------------------------------------------- softmax
    const int quad = warp & 3, r = quad * 32 + lane;
    const uint32_t tl = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const float c2 = a.scale * 1.4426950408889634f;
    const int pitch = kDh + kPartExtra;
    bool ok = true;
    int j = 0;
    for (Walk w(a, br); w.more() && ok; w.next(a)) {
      const int rows = w.gr.n * G, idx = w.tile * kPrefixRows + r;
      const bool used = w.tile * kPrefixRows + quad * 32 < rows;  // (some row of the warp)
      const int b = w.gr.first + min(idx, rows - 1) / G;
      const bool counts = idx < rows && a.lens[b] >= w.gr.prefix;
      float ref = -INFINITY, l = 0.0f;
      for (int ch = w.c0; ch < w.c1; ++ch, ++j) {
        const int st = j & 1, me = j & (kMetas - 1);
        const uint32_t ts = tl + kColS + kSCols * static_cast<uint32_t>(st);
        ok = mbar_wait_all(&br.meta_full[me], (j / kMetas) & 1, abort_flag, &g_prefix_wait_err);
        ok = ok && mbar_wait_all(&br.s_full[st], (j >> 1) & 1, abort_flag, &g_prefix_wait_err);
        if (!ok) break;
        tc_fence_after();
        if (used) {
          uint32_t valid[4];
          bool all = true;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            valid[i] = br.valid[me][i];
            all = all && valid[i] == 0xFFFFFFFFu;
          }
          if (!all && counts) {  // a page outside the cache, among the prefix's positions
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int left = w.gr.prefix - (ch * kPrefixChunk + 32 * i);
              const uint32_t want = left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
              if (want & ~valid[i]) atomicOr(&g_paged_err, kErrIndex);
            }
          }
          __syncwarp();
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t s[32];
            tmem_ld_32x32b_x32(ts + 32u * i, s);
            tmem_ld_wait();
            float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (valid[i] == 0xFFFFFFFFu) {
#pragma unroll
              for (int e = 0; e < 32; ++e) m4[e & 3] = fmaxf(m4[e & 3], __uint_as_float(s[e]) * c2);
            } else {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (valid[i] >> e & 1u) m4[e & 3] = fmaxf(m4[e & 3], __uint_as_float(s[e]) * c2);
            }
            top = fmaxf(top, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])));
          }
          float alpha = 1.0f;
          if (top > ref + kMove<kBf16>) {  // (-inf: the first score)
            alpha = exp2_fast(ref - top);
            ref = top;
            l *= alpha;
          }
          __syncwarp();
          const float from = ref == -INFINITY ? 0.0f : ref - kShift<kBf16>;
          float l4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            uint32_t s[32];
            tmem_ld_32x32b_x32(ts + 32u * i, s);
            tmem_ld_wait();
            uint32_t p01[32], p2[16];
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              float x0 = __uint_as_float(s[e]) * c2, x1 = __uint_as_float(s[e + 1]) * c2;
              if (valid[i] != 0xFFFFFFFFu) {
                if (!(valid[i] >> e & 1u)) x0 = -INFINITY;
                if (!(valid[i] >> e & 2u)) x1 = -INFINITY;
              }
              const float p0 = exp2_fast(x0 - from), p1 = exp2_fast(x1 - from);
              l4[e & 2] += p0;
              l4[(e & 2) + 1] += p1;
              uint32_t part[kPw];
              split2<kBf16>(p0, p1, part);
              p01[e / 2] = part[0];
              p01[16 + e / 2] = part[1];
              if constexpr (kBf16) p2[e / 2] = part[2];
            }
            tmem_st_x32(ts + 32u * i, p01);
            if constexpr (kBf16) tmem_st_x16(ts + 128u + 16u * i, p2);
          }
          l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
          // O of the unit's earlier chunks follows a moved reference, after their P V (the barrier of
          // chunk j - 1 cannot be a phase further: that is chunk j + 1's, which needs this warp's P)
          if (ch > w.c0 && __any_sync(0xFFFFFFFFu, alpha != 1.0f)) {
            ok = mbar_wait_all(&br.pv_done[(j - 1) & 1], ((j - 1) >> 1) & 1, abort_flag, &g_prefix_wait_err);
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < kDh / 32 && ok; ++i) {
              uint32_t o[32];
              tmem_ld_32x32b_x32(tl + 32u * i, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              tmem_st_x32(tl + 32u * i, o);
            }
          }
          tmem_st_wait();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&br.p_ready[st]);
        if (!ok) break;
      }
      if (!ok) break;
      // the part of the unit
      const int jl = j - 1;
      ok = mbar_wait_all(&br.pv_done[jl & 1], (jl >> 1) & 1, abort_flag, &g_prefix_wait_err);
      if (!ok) break;
      tc_fence_after();
      if (used) {
        const int h = w.hk * G + min(idx, rows - 1) % G;
        float* part = w.c0 == 0 ? a.parts + (static_cast<long long>(b) * a.H + h) * pitch
                                : a.parts + (static_cast<long long>(c.seqs) * a.H + static_cast<long long>(blockIdx.x) * kPrefixRows + r) * pitch;
#pragma unroll 1
        for (int i = 0; i < kDh / 32; ++i) {
          uint32_t o[32];
          __syncwarp();
          tmem_ld_32x32b_x32(tl + 32u * i, o);
          tmem_ld_wait();
          if (idx < rows) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(part + 32 * i + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        if (idx < rows) *reinterpret_cast<float2*>(part + kDh) = make_float2(ref, l);
        tc_fence_before();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&br.o_free);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_dealloc(tmem, kTmemCols);
}

template <bool kBf16, int kDh>
cudaError_t launch_prefix(const PrefixArgs& a, cudaStream_t stream, unsigned int* launches) {
  static SmemLimit limit;
  auto* kernel = prefix_kernel<kBf16, kDh>;
  cudaError_t e = limit.allow(kernel, smem_bytes<kDh>());
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(static_cast<unsigned>(a.grid)), dim3(kPrefixThreads), static_cast<size_t>(smem_bytes<kDh>()), stream, a);
  if (e != cudaSuccess) return e;
  ++*launches;
  const bool wide = a.H / a.kv.Hkv > 8, small = a.kv.page_log2 < 4;
  if (small)
    return wide ? launch<Rows<kBf16, kDh, true, true>, 2>(a, stream, launches) : launch<Rows<kBf16, kDh, true, true>, 1>(a, stream, launches);
  return wide ? launch<Rows<kBf16, kDh, false, true>, 2>(a, stream, launches) : launch<Rows<kBf16, kDh, false, true>, 1>(a, stream, launches);
}

size_t base_bytes(int groups) { return ((static_cast<size_t>(groups) + 1) * sizeof(unsigned long long) + 15) / 16 * 16; }

}  // namespace

size_t prefix_attention_workspace_bytes(int seqs, int groups, int H, int dh) {
  const size_t rows = static_cast<size_t>(seqs) * H + static_cast<size_t>(kMaxPrefixGrid) * kPrefixRows;
  return kWsBytes + base_bytes(groups) + rows * (dh + kPartExtra) * sizeof(float);
}

cudaError_t launch_prefix_attention(PrefixArgs a, cudaStream_t stream, unsigned int* launches) {
  uint8_t* ws = static_cast<uint8_t*>(a.ws) + kWsBytes;
  a.base = reinterpret_cast<unsigned long long*>(ws);
  a.parts = reinterpret_cast<float*>(ws + base_bytes(a.groups));
  a.grid = std::min(num_sms(), kMaxPrefixGrid);
  if (a.kv.bf16) return a.kv.dh == 64 ? launch_prefix<true, 64>(a, stream, launches) : launch_prefix<true, 128>(a, stream, launches);
  return a.kv.dh == 64 ? launch_prefix<false, 64>(a, stream, launches) : launch_prefix<false, 128>(a, stream, launches);
}

unsigned int prefix_read_and_clear_error() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_prefix_wait_err, sizeof(v));
  cudaMemcpyToSymbol(g_prefix_wait_err, &z, sizeof(z));
  return v;
}

unsigned int prefix_read_and_clear_index_error() { return read_and_clear_paged_error(); }

}  // namespace p4q
