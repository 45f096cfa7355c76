// Records of 4-bit weights and how they are expanded: what the kernels of the fully connected layers share (linear_q4.cu has the
// layout).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "mma_frag.cuh"

namespace gi {
namespace q4 {

using namespace frag;

constexpr int kUnitK = 128, kUnitWeights = kUnitK * 16 / 2;

// Masks of two weights of a word, and what they become the low digits of: operands out of a kernel's parameters (the compiler moves
// constants of this kind into registers again at every use).
struct Masks {
  unsigned low, high, digits;
};
inline Masks masks_of(int dtype) { return Masks{0x000f000fu, 0x00f000f0u, dtype == GI_F16 ? 0x64006400u : 0x43004300u}; }

// parts of a record that may belong to different groups
inline int parts_of(int group) { return group % 128 == 0 ? 1 : group % 64 == 0 ? 2 : 4; }
// Whether a layer's packed scales are 32 bits wide: those of 16 bits are kept where they are of the type its kernel computes in.
inline bool wide_scales(int scale_dtype, int dtype) { return scale_dtype != (dtype == GI_F16 ? static_cast<int>(GI_F16) : static_cast<int>(GI_BF16)); }

// Where an output's power of two brings its largest scale: in fp16 as far up as 15 times it allows, for the sake of the small ones.
inline int power_top(int dtype) { return dtype == GI_F16 ? 12 : 0; }

// bytes of a record, of what lies in front of its zero points
__host__ __device__ constexpr int zeros_at(int parts, bool wide) { return kUnitWeights + parts * 16 * (wide ? 4 : 2); }
__host__ __device__ constexpr int record_bytes(int parts, bool wide, bool zeros) {
  return (zeros_at(parts, wide) + (zeros ? parts * 16 : 0) + 31) / 32 * 32;  // whole sectors
}

__device__ __forceinline__ void copy16(unsigned dst, const void* src) {
  asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// all but the last N groups of this thread's copies have landed
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// What is subtracted from the digits of a word's rows g and g + 8.
struct Zero {
  unsigned lo, hi;
};
template <bool BF>
__device__ __forceinline__ Zero zero_of(const Masks& p, unsigned z_lo, unsigned z_hi) {
  if (BF) return Zero{p.digits | z_lo * 0x10001u, p.digits | z_hi * 0x10001u};  // 128 + z
  return Zero{p.digits | z_lo * 0x10001u, 0xd400d400u | z_hi * 0x100010u};      // 1024 + z, -(64 + z)
}

// Eight weights of a word as the A operand: q - z, exact.
template <bool BF>
__device__ __forceinline__ void expand(const Masks& p, unsigned w, const Zero& z, unsigned (&a)[4]) {
  if (BF) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned v = ((w >> (4 * i)) & p.low) | p.digits;  // 128 + q
      const unsigned c = i & 1 ? z.hi : z.lo;
      const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&c));
      a[i] = *reinterpret_cast<const unsigned*>(&d);
    }
  } else {
    const unsigned sixteenth = 0x2c002c00u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned u = i ? w >> 8 : w;
      const unsigned lo = (u & p.low) | p.digits;   // 1024 + q
      const unsigned hi = (u & p.high) | p.digits;  // 1024 + 16 q
      const __half2 d0 = __hsub2(*reinterpret_cast<const __half2*>(&lo), *reinterpret_cast<const __half2*>(&z.lo));
      const __half2 d1 = __hfma2(*reinterpret_cast<const __half2*>(&hi), *reinterpret_cast<const __half2*>(&sixteenth),
                                 *reinterpret_cast<const __half2*>(&z.hi));
      a[2 * i] = *reinterpret_cast<const unsigned*>(&d0);
      a[2 * i + 1] = *reinterpret_cast<const unsigned*>(&d1);
    }
  }
}

// Scales of rows g and g + 8.  S32: they are stored in 32 bits, else in the 16-bit type that x's kernel computes in (a choice by a
// value of the call, among all three types, took 21 instructions of a record's 130).
template <bool S32, bool BF>
__device__ __forceinline__ float2 load_scales(unsigned at) {
  if (S32) {
    const uint2 v = lds64(at);
    return make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
  }
  const unsigned v = lds32(at);
  if (BF) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
__device__ __forceinline__ unsigned lds16(unsigned at) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
  return v;
}

}  // namespace q4
}  // namespace gi
