// Rows by rows: 16 x 16 tiles of products between two sets of rows, both read
// along their contiguous dimension, for the kernels whose weights are plain
// row-major matrices.
//
// A k-step is 64 bytes of every row (32 bf16 or 16 float32 values): lane
// 16 g + c holds bytes 16 g .. 16 g + 15 of row c, one 16-byte load.  bf16 feeds
// one 16x16x32 instruction; float32 feeds four 16x16x4 ones, the j-th taking
// the j-th value of every lane, so that both operands agree on the order of k.
#pragma once

#include "fm_device.h"

namespace fm {

constexpr int kStepBytes = 64;

template <typename T>
__device__ __forceinline__ floatx4 mma_step(uint32x4 a, uint32x4 b, floatx4 c) {
  if constexpr (sizeof(T) == 2) {
    return mfma_bf16(__builtin_bit_cast(u16x8, a), __builtin_bit_cast(u16x8, b), c);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  }
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), static_cast<short>(0), static_cast<int>(bytes),
                                           kBufWord3);
}

// 16 bytes at `row + k`, or zeros where k lies past the row's end (k_end) or the
// row is kOutside.
__device__ __forceinline__ uint32x4 load_step(__amdgpu_buffer_rsrc_t rs, uint32_t row, uint32_t k, uint32_t k_end) {
  const uint32_t o = k < k_end && row != kOutside ? row + k : kOutside;
  return __builtin_amdgcn_raw_buffer_load_b128(rs, static_cast<int>(o), 0, 0);
}

}  // namespace fm
