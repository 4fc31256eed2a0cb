// Device-side layout and conversions of the paged 4-bit cache (include/kv4.h).
#pragma once

#include "kernel_common.h"

namespace attn {

// Bytes of a page (of 1 << shift tokens) of one head: the codes of K or V, their
// scales, and all of it.
template <int D>
__device__ __forceinline__ int kv4_code_bytes(int shift) { return (D / 2) << shift; }
template <int D>
__device__ __forceinline__ int kv4_scale_bytes(int shift) { return (D / 32) << shift; }
template <int D>
__device__ __forceinline__ int kv4_block_bytes(int shift) { return (D + D / 16) << shift; }

// Byte S of a word of codes as two packed 16-bit values times the power of two
// whose exponent `scale` has.  The instruction looks at the exponent bits of the
// scale alone, and gives NaN for 255.
template <typename T> struct Fp4;
template <> struct Fp4<_Float16> {
  template <int S>
  static __device__ __forceinline__ uint32_t cvt(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, S));
  }
};
template <> struct Fp4<__bf16> {
  template <int S>
  static __device__ __forceinline__ uint32_t cvt(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, S));
  }
};

}  // namespace attn
