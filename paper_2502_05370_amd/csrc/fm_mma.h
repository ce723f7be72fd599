// Rows by rows: 16 x 16 tiles of products between two sets of rows, both read
// along their contiguous dimension, for the kernels whose weights are plain
// row-major matrices.
//
// A k-step is 64 bytes of every row (32 bf16 or 16 float32 values), of which lane
// 16 g + c holds 16 bytes of row c.  bf16 feeds one 16x16x32 instruction; float32
// feeds four 16x16x4 ones, the j-th taking the j-th value of every lane.  Any
// assignment of the values of a row to k-steps and lane groups serves, as long
// as both operands agree on it.
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

// A group of two k-steps (128 bytes of every row) of 16 rows, loaded by two
// instructions: lane 16 g + c takes bytes 32 g + 16 (c % 2) .. + 15 of row c & ~1,
// then of row c | 1; the halves that belong to the neighbour lane's row change
// lanes in registers.  Two limits set this layout:
//   - A load serves one run of consecutive lanes with consecutive addresses, up to
//     64 bytes, per clock.  In the operands' own layout (a row per lane) a CU reads
//     38 GB/s from the L2, in pairs of lanes 76, in fours 150; HBM gives each of
//     256 CUs 28.
//   - HBM reaches its rate only where an instruction takes whole 128-byte lines,
//     and the streaming hint helps only then: 2 GB as 8 rows by 128 bytes with the
//     hint 7.0-7.2 TB/s, as 16 rows by 64 bytes 5.2-6.4 with or without it.
struct RowPairs {
  uint32_t even, odd;   // byte offsets of rows c & ~1 and c | 1 (or kOutside) with the lane's place
  static constexpr uint32_t kBytes = 2 * kStepBytes;
  RowPairs() = default;
  static __device__ __forceinline__ uint32_t place() {   // the lane's place in a row's 128 bytes
    const uint32_t lane = threadIdx.x % kWave;
    return lane / 16 * 32 + lane % 2 * 16;
  }
  // rows row0 .. row0 + 15 of `rows` rows of row_bytes from `base` on
  __device__ __forceinline__ RowPairs(int row0, int rows, uint32_t row_bytes, uint32_t base) {
    const int r = row0 + static_cast<int>(threadIdx.x % 16 / 2 * 2);
    even = r < rows ? base + static_cast<uint32_t>(r) * row_bytes + place() : kOutside;
    odd = r + 1 < rows ? base + static_cast<uint32_t>(r + 1) * row_bytes + place() : kOutside;
  }
  // 128 bytes from byte k (uniform) of the rows on; zeros from k_end on (a
  // multiple of 16).  k is the loads' scalar offset: a lane at kOutside stays
  // outside whatever k is, since the range check takes the scalar offset from the
  // buffer's size.
  template <int HINT>
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, uint32_t k, uint32_t k_end, uint32x4 (&v)[2]) const {
    const bool in = k + place() < k_end;
    const int ks = static_cast<int>(k < k_end ? k : 0u);
    v[0] = __builtin_amdgcn_raw_buffer_load_b128(rs, static_cast<int>(in ? even : kOutside), ks, HINT);
    v[1] = __builtin_amdgcn_raw_buffer_load_b128(rs, static_cast<int>(in ? odd : kOutside), ks, HINT);
  }
  // the operands of the two k-steps: bytes 32 g .. + 15 and 32 g + 16 .. + 31
  static __device__ __forceinline__ void steps(const uint32x4 (&v)[2], uint32x4 (&s)[2]) {
    const bool odd_lane = threadIdx.x % 2 != 0;
    constexpr int kFromEven = 0xA0, kFromOdd = 0xF5;   // lanes 0 0 2 2 and 1 1 3 3 of each four
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = __builtin_amdgcn_mov_dpp(v[1][i], kFromEven, 0xf, 0xf, true);
      const uint32_t b = __builtin_amdgcn_mov_dpp(v[0][i], kFromOdd, 0xf, 0xf, true);
      s[0][i] = odd_lane ? a : v[0][i];
      s[1][i] = odd_lane ? v[1][i] : b;
    }
  }
};
constexpr int kKeep = 0, kStream = 2;   // cache hints: read again soon, or once

}  // namespace fm
