// Attention of one new token per sequence over a paged key/value cache:
//   o_h = sum_{j < len} p_j v_j,  p = softmax_j(scale q_h . k_j).
//
// Work: a unit is one key/value head of one sequence with up to 8 NT of the
// query heads that share it (a group of more heads makes several units), cut
// into tiles of positions. Few units: each is a cluster's, and its CTAs'
// parts are added up in the first one's shared memory. Else all units' tiles in one
// row, unit after unit, are dealt to the CTAs in equal consecutive ranges, so a
// CTA's work does not depend on how unequal the sequences are (few tiles: one piece
// of a unit per CTA); the units that several CTAs share are joined by a second kernel.
//
// Bound: HBM. Times among other calls, on the GPU. 64 x 16384 positions, 32 heads over 8 of
// 128, bf16, pages of 16 (4.3 GB): 606 - 628 us = 6.8 - 7.1 TB/s, the measured copy (6.78); of
// 8 the same, of 1 727; of 64 dimensions 314 - 348 (pages of 8 381 - 390); 12 or 16 heads per key/value
// head, 4 of these, 353 (pages of 8 414: instructions). 24 sequences of up to 2048 x 40 heads 82 - 85 us
// = 0.92 of the copy, 128 of up to 8190 (skewed) x 8 167 - 171 = 0.96; one of 32011 x 8 28.4 = 0.68. Short ones
// cost a chain: lengths, page numbers, keys 4.6 us, then the end of a kernel and the second
// kernel 4, or the cluster's exchange 1.5: one of 704 x 40 6.2 us (by ranges 9.4), of 512 x 8
// 3.9 (6.9), 10 of 1024 x 8 11.0 (15.8).
#include "p4q_paged_kernel.cuh"
#include "p4q_paged_rows.cuh"

namespace p4q {
namespace {

template <bool kBf16, int kDh>
cudaError_t launch_for(const PagedAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  const bool wide = a.H / a.kv.Hkv > 8, small = a.kv.page_log2 < 4;
  if (small)
    return wide ? launch<Rows<kBf16, kDh, true>, 2>(a, stream, launches)
                : launch<Rows<kBf16, kDh, true>, 1>(a, stream, launches);
  return wide ? launch<Rows<kBf16, kDh, false>, 2>(a, stream, launches)
              : launch<Rows<kBf16, kDh, false>, 1>(a, stream, launches);
}

}  // namespace

size_t paged_attention_workspace_bytes() { return kWsBytes; }

int paged_clusters_at_once(DeviceNumber& known, SmemLimit& limit, const void* kernel, size_t smem, const cudaLaunchConfig_t& cfg) {
  int n = 0;
  const cudaError_t e = known.get(&n, [&](int* number) {
    const cudaError_t le = limit.allow(kernel, smem);
    if (le != cudaSuccess) return le;
    return cudaOccupancyMaxActiveClusters(number, kernel, &cfg);
  });
  if (e == cudaSuccess) return n;
  cudaGetLastError();
  return 0;
}

cudaError_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  if (a.kv.bf16) return a.kv.dh == 64 ? launch_for<true, 64>(a, stream, launches) : launch_for<true, 128>(a, stream, launches);
  return a.kv.dh == 64 ? launch_for<false, 64>(a, stream, launches) : launch_for<false, 128>(a, stream, launches);
}

unsigned int paged_read_and_clear_error() { return read_and_clear_paged_error(); }

}  // namespace p4q
