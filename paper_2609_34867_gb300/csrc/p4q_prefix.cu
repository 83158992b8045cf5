// Attention of one new token per sequence for groups of sequences that share a prefix: the
// prefix's keys and values are read once per group instead of once per sequence.
//
//   o = sum_i 2^(ref_i - ref) o_i / sum_i 2^(ref_i - ref) l_i
// over parts i of a sequence's positions, each with a reference ref_i, the sum l_i of the weights
// 2^(x_j - ref_i), x_j = scale log2(e) q . k_j, and the values o_i weighted so, all in fp32.
//
// Three kernels. prefix_kernel takes the prefixes: with n sequences of G query heads per
// key/value head there are n G rows of queries to the same keys, enough for the tensor cores'
// 128-row products (tcgen05 kind::f16, fp32 accumulators in TMEM). The paged attention kernel
// (p4q_paged_kernel.cuh) takes the positions that each sequence has of its own and leaves their
// parts. It needs nothing of the first, so it starts beside it, on what the first leaves free of the
// SMs. prefix_join_kernel adds the parts up and writes the outputs (inside the paged attention its
// waits held up the warps of all other units: 16 sequences behind 661 positions, 40 heads, 28.6 us,
// 21 this way).
//
// Bound: HBM where prefixes are long and their rows fill a tile or less (32 sequences behind 16384
// positions, 32 heads of 128, bf16: 119 us, 0.79 of what their bytes take); with several tiles per key head
// the softmax's chain, 3 us per chunk of 128 x 128 (64 sequences behind 4093, 32 heads over 8: 37 us of which
// bytes are 12.7); for short prefixes the chain of plan, queries and keys, chunk, end and join (21 us, bytes 4.5).
//
// prefix_kernel: units and ranges as p4q_paged_prefix.cuh says. Thirteen warps:
//   warps 0-3  queries, keys and values into shared memory with 16-byte asynchronous copies (pages
//              may be of any size and order, and positions past the prefix or of a page outside the
//              cache have to be zeros: 0 weight times an infinite value is NaN), in the 128-byte
//              swizzle that the products read; three stages of keys, two of values;
//   warps 4-11 two threads per row (its TMEM lane): scores' maximum, p = 2^(s - reference),
//              their sum, p as two fp16 or three bf16 values over the scores in TMEM; the
//              reference moves, and O with it, only when a score exceeds it by 2^4 (bf16 2^8);
//   warp 12    issues the products: S = Q K^T of the next chunk, then O += P V of this one, with
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

constexpr int kProducers = 4, kSoftmax = 8;          // warps
constexpr int kMmaWarp = kProducers + kSoftmax;
constexpr int kPrefixThreads = 32 * (kMmaWarp + 1);
// (more threads than there are: 80 registers for each, which leave 192 for each thread of one more warp on the quarter
// of the SM that has four of these: room for the own positions' kernel of up to 8 heads per key/value head (164 - 168),
// not for the one of more (210 - 252), which has what SMs without a CTA of the prefix leave it)
constexpr int kPrefixBound = 768;
constexpr int kMaxPrefixGrid = 160;
constexpr int kTileBytes = 16384;                    // 128 rows of 128 bytes
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 128, kSCols = 192;        // O: columns 0 .. 127; two S buffers, with room for P's third part
constexpr int kKStages = 3, kVStages = 2;            // (keys are wanted a chunk earlier than values)
constexpr int kMetas = 8;                            // of chunks' valid positions, see the producers

struct Bars {
  uint64_t q_full, q_empty, k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages], meta_full[kMetas];
  uint64_t s_full[2], p_ready[2], pv_done[2], o_free, mma_done;
  unsigned long long first, base, share, total;  // the CTA's range and the start of its first group
  int group;
  Group its;                                     // (that group)
  uint32_t valid[kMetas][kProducers];
  float sums[kPrefixRows];                       // of the second softmax warps' weights
  uint32_t tmem_slot;
  int abort_flag;
};

template <int kDh>
constexpr int smem_bytes() {
  return (kDh / 64) * kTileBytes * (1 + kKStages + kVStages) + static_cast<int>(sizeof(Bars)) + 1024;
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

__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// kind::f16 with fp16 or bf16 A and B (K-major; bit 16 set: B MN-major) and an fp32 accumulator, M x N.
template <bool kBf16>
constexpr uint32_t idesc16(int M, int N) {
  return (1u << 4) | (kBf16 ? (1u << 7) | (1u << 10) : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
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
  int copies;  // of the tile's rows, see the softmax
  __device__ Walk(const PrefixArgs& a, const Bars& br) : x(br.first), base(br.base), g(br.group) {
    end = min(br.total, x + br.share);
    if (x < end) {
      gr = br.its;
      find(a);
    }
  }
  __device__ bool more() const { return x < end; }
  __device__ void find(const PrefixArgs& a) {
    while (x >= base + group_chunks(a, gr)) {  // (x < total: such a group comes)
      base += group_chunks(a, gr);
      gr = load_group(a, ++g);
    }
    const unsigned int at = static_cast<unsigned int>(quotient(x - base, gr.chunks));
    c0 = static_cast<int>(x - base - static_cast<unsigned long long>(at) * gr.chunks);
    c1 = static_cast<int>(min(static_cast<unsigned long long>(gr.chunks), c0 + (end - x)));
    hk = static_cast<int>(at) / gr.tiles;
    tile = static_cast<int>(at) - hk * gr.tiles;
    const int rows = gr.n * (a.H / a.kv.Hkv) - tile * kPrefixRows;
    copies = copies_of(rows);
  }
  __device__ void next(const PrefixArgs& a) {
    x += c1 - c0;
    if (x < end) find(a);
  }
};

template <bool kBf16, int kDh>
__global__ void __launch_bounds__(kPrefixBound) prefix_kernel(const PrefixArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  constexpr int kHalves = kDh / 64;                 // 128-byte halves of a row
  constexpr int kOperand = kHalves * kTileBytes;
  constexpr int kOffK = kOperand, kOffV = kOffK + kKStages * kOperand, kOffBars = kOffV + kVStages * kOperand;
  constexpr int kPw = kParts<kBf16>;
  Bars& br = *reinterpret_cast<Bars*>(smem + kOffBars);
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  volatile int* const abort_flag = &br.abort_flag;
  const PagedCache& c = a.kv;
  const int G = a.H / c.Hkv;

  if (t == 0) {
    mbar_init(&br.q_full, 32 * kProducers);
    mbar_init(&br.q_empty, 1);
    for (int i = 0; i < kKStages; ++i) {
      mbar_init(&br.k_full[i], 32 * kProducers);
      mbar_init(&br.k_empty[i], 1);
    }
    for (int i = 0; i < kVStages; ++i) {
      mbar_init(&br.v_full[i], 32 * kProducers);
      mbar_init(&br.v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
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
  if (warp == kMmaWarp) {
    tmem_alloc(&br.tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_launch_dependents();
  if (warp == 0) {
    // the chunks before each group, their sum, and the group that the CTA's range begins in
    unsigned long long total = 0, last_begin = 0, last_end = 0;
    int most = 0;  // chunks of a unit
    Group gr = {};
    for (int g0 = 0; g0 < a.groups; g0 += 32) {
      const int g = g0 + lane;
      unsigned long long n = 0;
      if (g < a.groups) {
        gr = load_group(a, g);
        n = group_chunks(a, gr);
        if (n > 0) most = max(most, gr.chunks);
        if (blockIdx.x == 0 && (a.group_start[g] < 0 || a.group_start[g + 1] < a.group_start[g] ||
                                a.group_start[g + 1] > c.seqs || a.prefix_lens[g] > paged_room(c)))
          atomicOr(&g_paged_err, kErrIndex);
      }
      __syncwarp();
      const unsigned long long upto = total + scan_add(n);
      if (blockIdx.x == 0 && a.groups > 32 && g < a.groups) a.base[g] = upto - n;
      last_begin = upto - n;
      last_end = upto;
      total = __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    const unsigned long long share = prefix_share(total, most, a.grid), first = blockIdx.x * share;
    auto look = [&](int g, unsigned long long begin, unsigned long long end) {
      if (first >= begin && first < end) {
        br.group = g;
        br.base = begin;
        br.its = gr;
      }
    };
    if (a.groups <= 32) {
      look(lane, last_begin, last_end);
    } else {
      unsigned long long sum = 0;
      for (int g0 = 0; g0 < a.groups && sum <= first; g0 += 32) {
        const int g = g0 + lane;
        gr = g < a.groups ? load_group(a, g) : Group{};
        const unsigned long long n = g < a.groups ? group_chunks(a, gr) : 0;
        __syncwarp();
        const unsigned long long upto = sum + scan_add(n);
        look(g, upto - n, upto);
        sum = __shfl_sync(0xFFFFFFFFu, upto, 31);
      }
    }
    if (lane == 0) {
      if (blockIdx.x == 0) *a.share = share;
      br.first = first;
      br.share = share;
      br.total = total;
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
      const int idx = w.tile * kPrefixRows + (warp * 32 + lane & kPrefixRows / w.copies - 1);
      const uint16_t* qrow = nullptr;
      if (idx < w.gr.n * G)
        qrow = a.q + (w.gr.first + idx / G) * a.ldq + static_cast<long long>(w.hk * G + idx % G) * kDh;
      copy_rows(smem, qrow, a.q);
      cp_async_arrive(&br.q_full);
      for (int ch = w.c0; ch < w.c1; ++ch, ++j) {
        const int vs = j % kVStages, ks = j % kKStages;
        const int p = ch * kPrefixChunk + warp * 32 + lane;
        const bool valid = p < w.gr.prefix && static_cast<unsigned int>(page) < static_cast<unsigned int>(c.pages);
        const long long off = valid ? page * c.page_stride + (p & ((1 << c.page_log2) - 1)) * c.token_stride + w.hk * c.head_stride : 0;
        page = page_of(ch + 1);
        if (j >= kKStages) ok = mbar_wait_all(&br.k_empty[ks], (j / kKStages - 1) & 1, abort_flag, &g_prefix_wait_err);
        if (!ok) break;
        // Its place held those of chunk j - kMetas, which have been read: the product waited for here, S of chunk
        // j - kKStages, was issued behind P V of chunk j - kKStages - 2, and that one waited for the weights.
        static_assert(kMetas >= kKStages + 2, "valid positions");
        const uint32_t bits = __ballot_sync(0xFFFFFFFFu, valid);
        if (lane == 0) {
          br.valid[j & (kMetas - 1)][warp] = bits;
          mbar_arrive(&br.meta_full[j & (kMetas - 1)]);
        }
        copy_rows(smem + kOffK + ks * kOperand, valid ? c.k + off : nullptr, c.k);
        cp_async_arrive(&br.k_full[ks]);
        if (j >= kVStages) ok = mbar_wait_all(&br.v_empty[vs], (j / kVStages - 1) & 1, abort_flag, &g_prefix_wait_err);
        if (!ok) break;
        copy_rows(smem + kOffV + vs * kOperand, valid ? c.v + off : nullptr, c.v);
        cp_async_arrive(&br.v_full[vs]);
      }
    }
    cp_async_commit();
    cp_async_wait<0>();  // nothing of this CTA's copies may be in flight when it exits
  } else if (warp == kMmaWarp) {
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
      const int st = js & 1, ks = js % kKStages;
      if (cs == s.c0) ok = ok && mbar_wait_all(&br.q_full, us & 1, abort_flag, &g_prefix_wait_err);
      ok = ok && mbar_wait_all(&br.k_full[ks], (js / kKStages) & 1, abort_flag, &g_prefix_wait_err);
      if (!ok) return;
      fence_proxy_async_smem();  // the copies are seen by the products
      tc_fence_after();
      const uint32_t d = tmem + kColS + kSCols * static_cast<uint32_t>(st);
      const uint64_t b0 = k_desc + static_cast<uint32_t>(ks * (kOperand >> 4));
      const bool last = cs + 1 == s.c1;
      if (leader) {
#pragma unroll
        for (int kb = 0; kb < kHalves; ++kb)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_ss(d, q_desc + kb * (kTileBytes >> 4) + 2 * k, b0 + kb * (kTileBytes >> 4) + 2 * k, idS, (kb | k) != 0 ? 1u : 0u);
        mma_commit(&br.s_full[st]);
        mma_commit(&br.k_empty[ks]);
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
        const int st = j & 1, vs = j % kVStages;
        ok = ok && mbar_wait_all(&br.p_ready[st], (j >> 1) & 1, abort_flag, &g_prefix_wait_err);
        if (ch == w.c0 && uq > 0) ok = ok && mbar_wait_all(&br.o_free, (uq - 1) & 1, abort_flag, &g_prefix_wait_err);
        ok = ok && mbar_wait_all(&br.v_full[vs], (j / kVStages) & 1, abort_flag, &g_prefix_wait_err);
        if (!ok) break;
        fence_proxy_async_smem();
        tc_fence_after();
        const uint32_t pa = tmem + kColS + kSCols * static_cast<uint32_t>(st);
        const uint64_t b0 = v_desc + static_cast<uint32_t>(vs * (kOperand >> 4));
        if (leader) {
#pragma unroll
          for (int kt = 0; kt < kPrefixChunk / 16; ++kt)  // 16 positions per product: 8 columns of P, 16 rows of V
#pragma unroll
            for (int i = 0; i < kPw; ++i)
              mma_ts(tmem, pa + (i < 2 ? 16u * kt + 8u * i : 128u + 8u * kt), b0 + (2048 >> 4) * kt, idO,
                     (ch > w.c0 || kt > 0 || i > 0) ? 1u : 0u);
          mma_commit(&br.v_empty[vs]);
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
    // Two warps per 32 rows: both find the rows' maxima (which spares them an exchange), each makes the
    // weights of every other piece of 16 positions and has half of O's columns.
    // A tile of 32 rows and less stands in the products four times, of 64 and less twice; each copy
    // has weights for its share of a chunk's positions only, so that all warps work on them, and leaves
    // a part of its own. (For the others a copy has the least weights there are, not 0, which
    // would make NaN of an infinite value: 2^-34 of that at the reference in fp16, below 2^-124 in bf16.)
    constexpr uint32_t kNone = kBf16 ? 0x00800080u : 0x00010001u;
    constexpr int kPieces = kPrefixChunk / 16;
    const int quad = warp & 3, half = (warp - kProducers) >> 2, r = quad * 32 + lane;
    const uint32_t tl = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const float c2 = a.scale * 1.4426950408889634f;
    const float2 c22 = make_float2(c2, c2);
    const int pitch = kDh + kPartExtra;
    bool ok = true;
    int j = 0;
    // (After a failed wait a warp walks on without waits and work, so that the other one of its rows is
    // never left at their barrier.)
    for (Walk w(a, br); w.more(); w.next(a)) {
      const int per = kPrefixRows / w.copies, copy = r / per;  // rows of a copy
      const int rows = w.gr.n * G, idx = w.tile * kPrefixRows + (r & per - 1);
      const bool used = w.tile * kPrefixRows + (quad * 32 & per - 1) < rows;  // (some row of the warp)
      const int b = w.gr.first + min(idx, rows - 1) / G;
      const int i0 = copy * (kPieces / w.copies), i1 = i0 + kPieces / w.copies;  // its pieces
      float ref = -INFINITY, l = 0.0f;
      uint32_t lost = 0;
      for (int ch = w.c0; ch < w.c1; ++ch, ++j) {
        const int st = j & 1, me = j & (kMetas - 1);
        const uint32_t ts = tl + kColS + kSCols * static_cast<uint32_t>(st);
        ok = ok && mbar_wait_all(&br.meta_full[me], (j / kMetas) & 1, abort_flag, &g_prefix_wait_err);
        ok = ok && mbar_wait_all(&br.s_full[st], (j >> 1) & 1, abort_flag, &g_prefix_wait_err);
        tc_fence_after();
        if (used && !ok) named_bar_sync(1 + quad, 64);
        if (used && ok) {
          if (w.copies > 1) {  // other copies' pieces
            uint32_t none[16], none2[8];
#pragma unroll
            for (int e = 0; e < 16; ++e) none[e] = kNone;
#pragma unroll
            for (int e = 0; e < 8; ++e) none2[e] = kNone;
#pragma unroll 1
            for (int i = half; i < kPieces; i += 2)
              if (i < i0 || i >= i1) {
                tmem_st_x16(ts + 16u * i, none);
                if constexpr (kBf16) tmem_st_x8(ts + 128u + 8u * i, none2);
              }
          }
          const uint32_t* const valid = br.valid[me];
          const bool whole_chunk = (valid[0] & valid[1] & valid[2] & valid[3]) == 0xFFFFFFFFu;
          if (!whole_chunk) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // a page outside the cache, among the prefix's positions
              const int left = w.gr.prefix - (ch * kPrefixChunk + 32 * i);
              lost |= ~valid[i] & (left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u);
            }
          }
          float top = -INFINITY;
#pragma unroll 1
          for (int i = i0; i < i1; i += 2) {  // (an even number)
            uint32_t s[32];
            tmem_ld_32x32b_x32(ts + 16u * i, s);
            const uint32_t v = whole_chunk ? 0xFFFFFFFFu : valid[i >> 1];
            tmem_ld_wait();
            if (v != 0xFFFFFFFFu) {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (!(v >> e & 1u)) s[e] = 0x7FFFFFFFu;  // (NaN: no maximum)
            }
            if (!(c2 > 0.0f)) {
#pragma unroll
              for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(__fmul_rn(__uint_as_float(s[e]), c2));
            }
            float m4[4] = {top, top, top, top};
#pragma unroll
            for (int e = 0; e < 32; e += 2) m4[e >> 1 & 3] = max3(m4[e >> 1 & 3], __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
            top = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
          }
          // both warps have read all of their rows' scores: either overwrites only its own pieces with weights,
          // but the other one's maxima are of all
          if (c2 > 0.0f) top = __fmul_rn(top, c2);  // (rounding keeps the order: the largest product)
          named_bar_sync(1 + quad, 64);
          float alpha = 1.0f;
          if (top > ref + kMove<kBf16>) {  // (-inf: the first score)
            alpha = exp2_fast(ref - top);
            ref = top;
            l *= alpha;
          }
          __syncwarp();
          const float from = ref == -INFINITY ? 0.0f : ref - kShift<kBf16>;
          float2 l2[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll 1
          for (int i = i0 + half; i < i1; i += 2) {
            uint32_t s[16], p01[16], p2[8];
            tmem_ld_32x32b_x16(ts + 16u * i, s);
            const uint32_t v = whole_chunk ? 0xFFFFu : valid[i >> 1] >> (16 * (i & 1)) & 0xFFFFu;
            tmem_ld_wait();
            auto weights = [&](auto whole) {
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                // Scores are rounded as the reference is, before it is taken off: in one fma the largest would be off the
                // reference by half a place of fp32, which from 2^24 on is more than the powers have room for. (Two
                // sums: the compiler makes one fma of a packed product and a packed sum.)
                const float2 y = __fmul2_rn(make_float2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c22);
                float2 x = make_float2(__fsub_rn(y.x, from), __fsub_rn(y.y, from));
                if constexpr (!decltype(whole)::value) {
                  if (!(v >> e & 1u)) x.x = -INFINITY;
                  if (!(v >> e & 2u)) x.y = -INFINITY;
                }
                const float2 p = make_float2(exp2_fast(x.x), exp2_fast(x.y));
                l2[e >> 1 & 1] = __fadd2_rn(l2[e >> 1 & 1], p);
                uint32_t part[kPw];
                split2<kBf16>(p.x, p.y, part);
                p01[e / 2] = part[0];
                p01[8 + e / 2] = part[1];
                if constexpr (kBf16) p2[e / 2] = part[2];
              }
            };
            if (v == 0xFFFFu)
              weights(std::true_type{});
            else
              weights(std::false_type{});
            __syncwarp();
            tmem_st_x16(ts + 16u * i, p01);
            if constexpr (kBf16) tmem_st_x8(ts + 128u + 8u * i, p2);
          }
          l += (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
          // O of the unit's earlier chunks follows a moved reference, after their P V (the barrier of
          // chunk j - 1 cannot be a phase further: that is chunk j + 1's, which needs this warp's P)
          if (ch > w.c0 && __any_sync(0xFFFFFFFFu, alpha != 1.0f)) {
            ok = mbar_wait_all(&br.pv_done[(j - 1) & 1], ((j - 1) >> 1) & 1, abort_flag, &g_prefix_wait_err);
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < kDh / 64 && ok; ++i) {
              uint32_t o[32];
              const uint32_t at = tl + static_cast<uint32_t>(kDh / 2 * half + 32 * i);
              tmem_ld_32x32b_x32(at, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              tmem_st_x32(at, o);
            }
          }
          tmem_st_wait();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&br.p_ready[st]);
      }
      if (lost != 0 && idx < rows && a.lens[b] >= w.gr.prefix) atomicOr(&g_paged_err, kErrIndex);
      __syncwarp();
      // the part of the unit
      const int jl = j - 1;
      ok = ok && mbar_wait_all(&br.pv_done[jl & 1], (jl >> 1) & 1, abort_flag, &g_prefix_wait_err);
      tc_fence_after();
      const int h = w.hk * G + min(idx, rows - 1) % G;
      const long long all = static_cast<long long>(c.seqs) * a.H;
      float* const part = a.parts + pitch * (w.c0 == 0 ? copy * all + static_cast<long long>(b) * a.H + h
                                                       : kCopies * all + static_cast<long long>(blockIdx.x) * kPrefixRows + r);
      if (used && ok) {
#pragma unroll 1
        for (int i = 0; i < kDh / 64; ++i) {
          uint32_t o[32];
          const int at = kDh / 2 * half + 32 * i;
          __syncwarp();
          tmem_ld_32x32b_x32(tl + static_cast<uint32_t>(at), o);
          tmem_ld_wait();
          if (idx < rows) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(part + at + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        tc_fence_before();
      }
      // The sum of both warps' pieces. (One of them writes it: a part's last four floats by both as ref, l0 and l1 took
      // 1 - 3 us: 4 sequences behind 30000 28.3 instead of 25.0, five documents 29.6 instead of 28.1.)
      if (used) {
        if (half == 1) br.sums[r] = l;
        named_bar_sync(1 + quad, 64);
        if (ok && half == 0 && idx < rows)
          *reinterpret_cast<float4*>(part + kDh) = make_float4(ref, l + br.sums[r], 0.0f, 0.0f);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&br.o_free);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

// Adds up the parts of every head of every sequence: kWarpsPer warps per head (dh 64: two heads at once), each every
// kWarpsPer-th part, eight of them on their way together.
constexpr int kJoinThreads = 128;

template <bool kBf16, int kDh, int kWarpsPer>
__global__ void __launch_bounds__(kJoinThreads) prefix_join_kernel(const PrefixArgs a) {
  constexpr int kLanes = kDh / 4, kSides = 32 / kLanes, kRows = kJoinThreads / 32 / kWarpsPer * kSides, kBatch = 8;
  constexpr int kPitch = kDh + kPartExtra;
  __shared__ float4 so[kJoinThreads / 32][32];
  __shared__ float2 sml[kJoinThreads / 32][kSides];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, side = lane / kLanes, d = lane % kLanes * 4;
  const int rows = a.kv.seqs * a.H;  // (fits in 31 bits)
  const int at = static_cast<int>(blockIdx.x) * kRows + warp / kWarpsPer * kSides;
  const int row = min(at + side, rows - 1);  // (all warps stay, for their barrier)
  const int G = a.H / a.kv.Hkv, b0 = min(at, rows - 1) / a.H, b = kSides > 1 ? row / a.H : b0, h = row - b * a.H;
  see_earlier_kernels();
  PrefixOf of(a, b0, a.lens[b0]);
  if (kSides > 1) {  // (the second of two heads may be the next sequence's first)
    const int b1 = min(at + kSides - 1, rows - 1) / a.H;
    if (b1 != b0) {
      const PrefixOf other(a, b1, a.lens[b1]);
      if (side == 1) of = other;
    }
  }
  pdl_wait();
  pdl_launch_dependents();
  int parts = 0, c0 = 0, copies_log2 = 0, lane_row = 0;
  if (of.g >= 0) {
    const Group& r = of.r;
    const unsigned long long share = *a.share;
    const int hk = h / G, i = (b - r.first) * G + h - hk * G;
    const unsigned long long x = (a.groups > 32 ? a.base[of.g] : of.begin) + static_cast<unsigned long long>(hk * r.tiles + i / kPrefixRows) * r.chunks;
    c0 = min(static_cast<int>(quotient(x, share)), a.grid - 1);
    const int c1 = min(static_cast<int>(quotient(x + r.chunks - 1, share)), a.grid - 1);
    copies_log2 = copies_of(r.n * G - i / kPrefixRows * kPrefixRows) >> 1;  // (of 1, 2, 4)
    lane_row = i % kPrefixRows;
    parts = (c1 - c0 + 1) << copies_log2;
  }
  const float* const own = a.own + static_cast<long long>(row) * kPitch;
  const float* const first = a.parts + static_cast<long long>(row) * kPitch;
  const float* const more = a.parts + (kCopies * static_cast<long long>(rows) + lane_row) * kPitch;
  float top = -INFINITY, sum = 0.0f;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  // part 0 is that of the sequence's own positions
  for (int k = warp % kWarpsPer; k <= parts; k += kBatch * kWarpsPer) {
    float pm[kBatch], pl[kBatch];
    float4 pv[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int n = k + i * kWarpsPer;
      pm[i] = -INFINITY;
      pl[i] = 0.0f;
      pv[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (n <= parts) {
        const int c = (n - 1) >> copies_log2, copy = (n - 1) & ((1 << copies_log2) - 1);
        const float* p = n == 0   ? own
                         : c == 0 ? first + copy * static_cast<long long>(rows) * kPitch
                                  : more + (static_cast<long long>(c0 + c) * kPrefixRows + copy * (kPrefixRows >> copies_log2)) * kPitch;
        const float2 ml = *reinterpret_cast<const float2*>(p + kDh);
        pm[i] = ml.x;
        pl[i] = ml.y;
        pv[i] = *reinterpret_cast<const float4*>(p + d);
      }
    }
    const float old = top;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) top = fmaxf(top, pm[i]);
    const float f = old == -INFINITY ? 0.0f : exp2_fast(old - top);
    sum *= f;
    v.x *= f;
    v.y *= f;
    v.z *= f;
    v.w *= f;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float e = pm[i] == -INFINITY ? 0.0f : exp2_fast(pm[i] - top);  // (of NaN sums 0 makes NaN)
      sum += pl[i] * e;
      if (e != 0.0f) {  // (a copy without positions has infinite values where others have)
        v.x += pv[i].x * e;
        v.y += pv[i].y * e;
        v.z += pv[i].z * e;
        v.w += pv[i].w * e;
      }
    }
  }
  if (kWarpsPer > 1) {
    so[warp][lane] = v;
    if (d == 0) sml[warp][side] = make_float2(top, sum);
    __syncthreads();
    if (warp % kWarpsPer != 0) return;
    const float mine = top;
#pragma unroll
    for (int w = 1; w < kWarpsPer; ++w) top = fmaxf(top, sml[warp + w][side].x);
    const float f = mine == -INFINITY ? 0.0f : exp2_fast(mine - top);
    sum *= f;
    if (f == 0.0f) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    v.x *= f;
    v.y *= f;
    v.z *= f;
    v.w *= f;
#pragma unroll
    for (int w = 1; w < kWarpsPer; ++w) {
      const float2 ml = sml[warp + w][side];
      const float e = ml.x == -INFINITY ? 0.0f : exp2_fast(ml.x - top);
      const float4 z = so[warp + w][lane];
      sum += ml.y * e;
      if (e != 0.0f) {
        v.x += z.x * e;
        v.y += z.y * e;
        v.z += z.z * e;
        v.w += z.w * e;
      }
    }
  }
  if (at + side >= rows) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint2 w = make_uint2(pack2<kBf16>(v.x * inv, v.y * inv), pack2<kBf16>(v.z * inv, v.w * inv));
  if (sum == 0.0f) w = make_uint2(0u, 0u);
  *reinterpret_cast<uint2*>(a.o + b * a.ldo + static_cast<long long>(h) * kDh + d) = w;
  if (d == 0 && a.lse) a.lse[row] = sum == 0.0f ? -INFINITY : (top - kShift<kBf16>) * 0.6931471805599453f + logf(sum);
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
    e = wide ? launch<Rows<kBf16, kDh, true, true>, 2>(a, stream, launches) : launch<Rows<kBf16, kDh, true, true>, 1>(a, stream, launches);
  else
    e = wide ? launch<Rows<kBf16, kDh, false, true>, 2>(a, stream, launches) : launch<Rows<kBf16, kDh, false, true>, 1>(a, stream, launches);
  if (e != cudaSuccess) return e;
  // four warps per head, of many heads two (us, with four, two, one: 64 x 32 heads of 6 parts 39.4, 36.9, 36.7; 96 x 24 of
  // 64 dimensions and up to 20 28.7, 28.8, 29.4; 32 x 32 of up to 4 119.7, 120.6, 121.3; 4 x 8 of 120 24.6, 28.9, 37.9)
  const long long rows = static_cast<long long>(a.kv.seqs) * a.H;
  constexpr int kSides = kDh == 64 ? 2 : 1;
  const bool few = rows <= 8ll * num_sms();
  const long long per = (few ? 1 : 2) * kSides;  // rows of a CTA
  e = launch_pdl(few ? prefix_join_kernel<kBf16, kDh, 4> : prefix_join_kernel<kBf16, kDh, 2>,
                 dim3(static_cast<unsigned>((rows + per - 1) / per)), dim3(kJoinThreads), 0, stream, a);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace

size_t prefix_attention_workspace_bytes(int seqs, int groups, int H, int dh) {
  const size_t rows = (kCopies + 1) * static_cast<size_t>(seqs) * H + static_cast<size_t>(kMaxPrefixGrid) * kPrefixRows;
  return rows * (dh + kPartExtra) * sizeof(float) + (2 + static_cast<size_t>(groups)) * sizeof(unsigned long long);
}

cudaError_t launch_prefix_attention(PrefixArgs a, cudaStream_t stream, unsigned int* launches) {
  const size_t rows = static_cast<size_t>(a.kv.seqs) * a.H;
  a.own = static_cast<float*>(a.ws);
  a.parts = a.own + rows * (a.kv.dh + kPartExtra);
  a.share = reinterpret_cast<unsigned long long*>(
      a.parts + (kCopies * rows + static_cast<size_t>(kMaxPrefixGrid) * kPrefixRows) * (a.kv.dh + kPartExtra));
  a.base = a.share + 1;
  // Heads of 128: half of the SMs. The others are the own positions' kernel's from the beginning; an SM that has run a
  // CTA of the prefix keeps its 200 KB of shared memory and leaves that kernel's loads little of L1, so CTAs that
  // end at once are no better than few. us, on half, three quarters and all of the SMs: 64 conversations behind 4093
  // positions 40.7, 45.8, 45.7; 32 behind 16384 121.6, 127.5, 137.6; 16 questions about one image 20.1, 20.0,
  // 21.8. Of 64 a CTA has half as much: five documents 36.0, 31.9, 30.0.
  a.grid = std::min(a.kv.dh == 64 ? num_sms() : num_sms() / 2, kMaxPrefixGrid);
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
