// What a launch needs of its device, asked or set once on each: dynamic shared
// memory past 48 KB has to be allowed for a kernel before it is launched with it,
// and what fits at once is the device's to say.
#pragma once

#include <atomic>
#include <cstdint>
#include <cuda_runtime_api.h>

namespace p4q {

// One per kernel, beside its launch. allow() sets the kernel's limit on the
// current device, the first time that it is called there; bytes is the largest
// that any launch asks for, so that threads that set it together set the same.
class SmemLimit {
 public:
  template <class Kernel>
  cudaError_t allow(Kernel* kernel, size_t bytes) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;  // further devices: set on every call
    if (done_.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(bytes));
    if (e == cudaSuccess) done_.fetch_or(bit, std::memory_order_relaxed);
    return e;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

// A number that the runtime tells about the current device (clusters that fit at
// once), asked the first time that it is wanted there. A question that failed is
// asked again the next time.
class DeviceNumber {
 public:
  template <class Ask>  // cudaError_t ask(int* number)
  cudaError_t get(int* number, Ask&& ask) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool kept = dev >= 0 && dev < kDevices;  // further devices: asked on every call
    if (kept) {
      const int known = known_[dev].load(std::memory_order_relaxed);
      if (known > 0) {
        *number = known - 1;
        return cudaSuccess;
      }
    }
    e = ask(number);
    if (e == cudaSuccess && kept) known_[dev].store(*number + 1, std::memory_order_relaxed);
    return e;
  }

 private:
  static constexpr int kDevices = 64;
  std::atomic<int> known_[kDevices] = {};  // one more than the number; 0: not asked yet
};

}  // namespace p4q
