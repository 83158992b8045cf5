// What the attention over a paged cache is made of, whatever the cache holds: the
// tensor-core product, the exponential, and what a unit of work is.
#pragma once

#include <cuda_runtime.h>

#include "p4q_device.cuh"
#include "p4q_elem.cuh"
#include "p4q_internal.h"

namespace p4q {

namespace {
__device__ unsigned int g_paged_err;  // one for each source file that includes this
}  // namespace

namespace paged {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;

template <bool kBf16>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if (kBf16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// A shared-memory load that stays where it is (not hoisted out of a loop).
__device__ __forceinline__ uint4 reload16(const uint4* p) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem_u32(p)));
  return v;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// For a kernel that reads what the stream's earlier kernels wrote without waiting for the one before it, which writes
// none of that: the one before has waited for all of them (griddepcontrol.wait: they are complete, and what they
// wrote is performed) before it let this one begin, in every thread of its CTAs; what this SM's L1 may still have of their data
// from before is given up here. What it rests on: a launch that griddepcontrol.launch_dependents releases is
// promised no sight of anything by itself; that it begins behind the instruction that released it, and
// that the fence drops this SM's older lines, is what makes it see writes performed before.
__device__ __forceinline__ void see_earlier_kernels() { __threadfence(); }

// What a unit is to the part of the kernel that goes through its tiles: heads h0 ..
// h0 + heads - 1 of sequence b over key/value head hk, positions from .. len - 1
// (from is 0 but where a prefix is another kernel's), tiles counted from base.
struct Unit {
  const int32_t* table;
  int b, hk, h0, heads, len, from, base;
};

// Of a sequence whose positions are all the kernel's own.
struct NoPrefix {
  static constexpr int from = 0;
  int row;
  template <class Args>
  __device__ __forceinline__ NoPrefix(const Args&, int b, int) : row(b) {}
};

// A warp's part of a unit: O^T ([.][hh][j]: dimensions C::first_dim(hh, g) + 2 j (+ 1),
// heads 2 t, 2 t + 1), the references and the sums.
template <int kNt, int kVc>
struct Part {
  float o[kNt][kVc][4][4];
  float ref[kNt][2], l[kNt][2];
};

}  // namespace paged
}  // namespace p4q
