// Arguments of the norms around a block (fm_norm.hip).
#pragma once

#include <type_traits>

#include "fm_internal.h"

namespace fm {

struct NormArgs {
  const void* x;      // [T][d]
  const void* y;      // [T][d] or null
  const void* post;   // [d] or null
  const void* gate;   // by kind, or null
  const void* pre;    // [d] or null
  int32_t gate_kind;
  float scale, eps;
  int32_t T, d;
  void* r_out;        // or null
  void* h_out;
};
hipError_t launch_norm(const NormArgs& a, fm_dtype dt, hipStream_t st);

struct NormGradArgs {
  NormArgs f;         // the forward call's, without its outputs
  const void* dr;     // [T][d] or null
  const void* dh;     // [T][d] or null
  int32_t accumulate;
  void* dx;
  void* dy;
  float* dpost;
  void* dgate;
  float* dpre;
  float* partial;     // [lists][2][d]
};
constexpr int kNormLists = 256;   // partial sums at most: a workgroup on every CU
size_t norm_scratch_bytes(int32_t T_max, int32_t d);
hipError_t launch_norm_grad(const NormGradArgs& a, fm_dtype dt, hipStream_t st);

}  // namespace fm
