// Attention of one new token per sequence over a paged cache of 8- or 4-bit codes.
#include "p4q_paged_kernel.cuh"
#include "p4q_paged_codes.cuh"

namespace p4q {
namespace {

template <int kBits, int kDh>
cudaError_t launch_for(const QuantAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  const int group = a.H / a.kv.Hkv;
  const bool small = a.kv.page_log2 < 4;
  if (group <= 4)
    return small ? launch<Codes<kBits, kDh, true, true>, 1>(a, stream, launches) : launch<Codes<kBits, kDh, false, true>, 1>(a, stream, launches);
  if (group <= 8)
    return small ? launch<Codes<kBits, kDh, true, false>, 1>(a, stream, launches) : launch<Codes<kBits, kDh, false, false>, 1>(a, stream, launches);
  return small ? launch<Codes<kBits, kDh, true, false>, 2>(a, stream, launches) : launch<Codes<kBits, kDh, false, false>, 2>(a, stream, launches);
}

}  // namespace

cudaError_t launch_paged_attention_quant(const QuantAttnArgs& a, cudaStream_t stream, unsigned int* launches) {
  if (a.kv.bits == 8) return a.kv.dh == 64 ? launch_for<8, 64>(a, stream, launches) : launch_for<8, 128>(a, stream, launches);
  return a.kv.dh == 64 ? launch_for<4, 64>(a, stream, launches) : launch_for<4, 128>(a, stream, launches);
}

unsigned int paged_quant_read_and_clear_error() { return read_and_clear_paged_error(); }

}  // namespace p4q
