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

// A group of two k-steps (128 bytes of every row) of 16 weight rows, streamed
// once.  HBM reaches its rate only where each load instruction takes whole
// 128-byte lines, and the streaming hint helps it only then: reading 2 GB as 8
// rows by 128 bytes with the hint runs at 7.0-7.2 TB/s on an MI355X, as 16 rows by
// 64 bytes, the operands' own layout, at 5.2-6.4 TB/s with or without it.  So lane
// 16 g + c loads 16 bytes at 64 (c / 8) + 16 g of row c % 8 and of row 8 + c % 8,
// and the halves that belong to the other k-step change lanes c <-> c ^ 8.
struct WeightRows {
  uint32_t lo, hi;   // byte offsets of rows c % 8 and 8 + c % 8 (or kOutside), with the lane's place in the line
  uint32_t lane_k;   // that place
  WeightRows() = default;
  __device__ __forceinline__ WeightRows(int row0, int rows, uint32_t row_bytes, uint32_t base, int c, int g) {
    lane_k = static_cast<uint32_t>(c / 8) * kStepBytes + static_cast<uint32_t>(g) * 16u;
    const int r = row0 + c % 8;
    lo = r < rows ? base + static_cast<uint32_t>(r) * row_bytes + lane_k : kOutside;
    hi = r + 8 < rows ? base + static_cast<uint32_t>(r + 8) * row_bytes + lane_k : kOutside;
  }
  // the lines at byte k of the rows; zeros from k_end on
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, uint32_t k, uint32_t k_end, uint32x4 (&v)[2]) const {
    constexpr int kStream = 2;
    const bool in = k + lane_k < k_end;
    v[0] = __builtin_amdgcn_raw_buffer_load_b128(rs, static_cast<int>(in && lo != kOutside ? lo + k : kOutside), 0, kStream);
    v[1] = __builtin_amdgcn_raw_buffer_load_b128(rs, static_cast<int>(in && hi != kOutside ? hi + k : kOutside), 0, kStream);
  }
  // the operands of the group's two k-steps
  static __device__ __forceinline__ void steps(const uint32x4 (&v)[2], uint32x4 (&s)[2]) {
    constexpr int kRor8 = 0x128;   // lanes c <-> c ^ 8 of each 16
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[0][i] = __builtin_amdgcn_update_dpp(v[0][i], v[1][i], kRor8, 0xf, 0xc, false);   // lanes 8..15 from v[1]
      s[1][i] = __builtin_amdgcn_update_dpp(v[1][i], v[0][i], kRor8, 0xf, 0x3, false);   // lanes 0..7 from v[0]
    }
  }
};

}  // namespace fm
