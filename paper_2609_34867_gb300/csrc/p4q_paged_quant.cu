// Attention of one new token per sequence over a paged cache of 8- or 4-bit codes: the instances of the
// paged attention kernel with p4q_paged_codes.cuh's way through a unit's tiles, and which call takes which.
#include "p4q_paged_kernel.cuh"
#include "p4q_paged_codes.cuh"

namespace p4q {
namespace {

template <int kBits, int kDh, bool kSmall>
cudaError_t launch_for(const QuantAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  const int group = a.H / a.kv.Hkv;
  // 8-bit rows of 64 bytes: two heads of a line of HBM to a CTA (64 sequences of up to 4096 x 40 heads of 64
  // 135 us, on other GPUs to 144; on the first, with one head to a CTA, fetched as half lines 165, as whole ones 141). 4-bit codes are bound by instructions before
  // that, and finer units are better (128 of up to 8190 x 8 heads 79.5 us, two to a CTA 84.8).
  constexpr bool kTwo = kBits == 8 && kDh == 64;
  if (kTwo && a.kv.Hkv % 2 == 0 && group <= 8)
    return group <= 4 ? launch<Codes<kBits, kDh, kSmall, true, kTwo ? 2 : 1>, 1>(a, stream, launches)
                      : launch<Codes<kBits, kDh, kSmall, false, kTwo ? 2 : 1>, 1>(a, stream, launches);
  if (group <= 4) return launch<Codes<kBits, kDh, kSmall, true, 1>, 1>(a, stream, launches);
  return group <= 8 ? launch<Codes<kBits, kDh, kSmall, false, 1>, 1>(a, stream, launches)
                    : launch<Codes<kBits, kDh, kSmall, false, 1>, 2>(a, stream, launches);
}

template <int kBits, int kDh>
cudaError_t launch_for(const QuantAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  return a.kv.page_log2 < 4 ? launch_for<kBits, kDh, true>(a, stream, launches) : launch_for<kBits, kDh, false>(a, stream, launches);
}

}  // namespace

cudaError_t launch_paged_attention_quant(const QuantAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  if (a.kv.bits == 8) return a.kv.dh == 64 ? launch_for<8, 64>(a, stream, launches) : launch_for<8, 128>(a, stream, launches);
  return a.kv.dh == 64 ? launch_for<4, 64>(a, stream, launches) : launch_for<4, 128>(a, stream, launches);
}

unsigned int paged_quant_read_and_clear_error() { return read_and_clear_paged_error(); }

}  // namespace p4q
