// The chosen experts' products of one MoE layer for the few tokens of a decode
// iteration, on experts that sit in the slots of an expert cache.
//
//   h[t,e]  = weight(t,e) * silu(Gate_e x[t]) * (Up_e x[t])
//   out[t]  = residual[t] + sum over e of Down_e h[t,e]
//
// With few tokens each weight meets a handful of columns, so reading every
// expert in use once from HBM bounds both products (6 T K d f operations on
// 6 d f bytes per expert in bf16).  Two launches: k_moe_up (Gate and Up, joined
// to h) and k_moe_down.  Weights go straight from memory to the registers of
// the matrix instructions, 16 rows by 128 contiguous bytes per load group;
// activations, the other operand, come from the caches.  The wavefronts of a
// workgroup split the long axis, which keeps many loads in flight for any
// number of experts, and their sums meet in LDS in a fixed order.
//
// h keeps 16 bits of mantissa in bf16 models: it is stored as the nearest bf16
// and the nearest bf16 of the rest, both multiplied, so that the only rounding
// to bf16 that shows is the output's own.  The weights' stream bounds the
// second product, and the extra matrix instructions hide behind it.
#include <type_traits>

#include "fm_internal.h"
#include "fm_mma.h"

namespace fm {

namespace {

constexpr int kUpWaves = 8;
constexpr int kUpRows = 16;        // rows of Gate and of Up per workgroup
constexpr int kMaxSplits = 16;     // workgroups that share one block of output rows
constexpr int kGroupBytes = 2 * kStepBytes;   // of every row in one load group

struct MoeArgs {
  const char* slots;
  const int32_t* slot_of;
  const char* x;             // [T][d] of this launch's tokens
  const int32_t* ids;        // [T][K]
  const float* weight;       // [T][K]
  const char* residual;      // [T][d] or null
  char* out;                 // [T][d]
  char* h;                   // [T * K][f]: float32, or bf16 with the rest's plane after it
  float* partial;            // [splits][T][d]
  uint32_t* ticket;          // [row blocks of the output]
  uint32_t* flags;
  int32_t T, K, E, n_slots, d, f, splits, row_blocks;
};

// Which tokens take which experts, in LDS: for every expert in use its slot,
// its number of tokens and the first of its places in the concatenated lists.
struct Plan {
  uint64_t takes[kMaxE][kMoeTokens / 64];   // tokens that take the expert
  int32_t slot[kMaxE];
  int32_t count[kMaxE];
  int32_t first[kMaxE];
  int32_t used[kMaxE];      // the experts in use, in order
  int32_t n_used;
};

// Filled by the whole workgroup; ends with a barrier.
__device__ __forceinline__ void make_plan(const MoeArgs& a, Plan& pl) {
  const int tid = threadIdx.x;
  for (int i = tid; i < kMaxE * (kMoeTokens / 64); i += blockDim.x) pl.takes[i / (kMoeTokens / 64)][i % (kMoeTokens / 64)] = 0;
  if (tid < kMaxE) pl.slot[tid] = tid < a.E ? a.slot_of[tid] : -1;
  __syncthreads();
  uint32_t bad = 0;
  for (int i = tid; i < a.T * a.K; i += blockDim.x) {
    const int e = a.ids[i];
    if (e < 0) continue;
    const int s = e < a.E ? pl.slot[e] : 0;
    if (e >= a.E || s >= a.n_slots) {
      bad |= FM_FLAG_INDEX_RANGE;
    } else if (s < 0) {
      bad |= FM_FLAG_EXPERT_MISSING;
    } else {
      const int t = i / a.K;
      atomicOr(reinterpret_cast<unsigned long long*>(&pl.takes[e][t / 64]), 1ull << (t % 64));
    }
  }
  if (bad != 0 && a.flags != nullptr && blockIdx.x == 0) atomicOr(a.flags, bad);
  __syncthreads();
  if (tid < kWave) {
    int n = 0;
#pragma unroll
    for (int j = 0; j < kMoeTokens / 64; ++j) n += __popcll(pl.takes[tid][j]);
    int incl = n;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int v = __shfl_up(incl, o, kWave);
      if (tid >= o) incl += v;
    }
    const uint64_t in_use = __ballot(n > 0);
    pl.count[tid] = n;
    pl.first[tid] = incl - n;
    if (n > 0) pl.used[__popcll(in_use & ((1ull << tid) - 1ull))] = tid;
    if (tid == 0) pl.n_used = __popcll(in_use);
  }
  __syncthreads();
}

// Place of token t among the tokens that take expert e (t takes it).
__device__ __forceinline__ int place_of(const Plan& pl, int e, int t) {
  int n = 0;
  for (int j = 0; j < t / 64; ++j) n += __popcll(pl.takes[e][j]);
  return n + __popcll(pl.takes[e][t / 64] & ((1ull << (t % 64)) - 1ull));
}
__device__ __forceinline__ bool takes(const Plan& pl, int e, int t) { return (pl.takes[e][t / 64] >> (t % 64)) & 1ull; }

__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }

// ---------------------------------------------------------------- gate and up

// One pass over a block of 16 gate and 16 up rows for up to 16 N of the
// expert's tokens.  The wavefronts deal the load groups of a row among
// themselves, starting at a place that differs from block to block: rows of a
// power of two bytes would otherwise keep all workgroups on few memory channels
// at a time (2 GB in rows of 8 KB: 5.9 -> 7.1 TB/s).
template <typename T, int N, int PA>
__device__ __forceinline__ void up_pass(const MoeArgs& a, __amdgpu_buffer_rsrc_t rs_w, __amdgpu_buffer_rsrc_t rs_x,
                                        int row0, const int32_t* tok, const float* wt, int n, int place0,
                                        floatx4 (*red)[2][N][kWave]) {
  const int lane = threadIdx.x % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane % 16;
  const int g = lane / 16;
  const uint32_t rb = static_cast<uint32_t>(a.d) * sizeof(T);
  const WeightRows w_gate(row0, a.f, rb, 0u, c, g);
  const WeightRows w_up(row0, a.f, rb, static_cast<uint32_t>(a.f) * rb, c, g);
  uint32_t ro_x[N];
#pragma unroll
  for (int j = 0; j < N; ++j) ro_x[j] = 16 * j + c < n ? static_cast<uint32_t>(tok[16 * j + c]) * rb : kOutside;
  floatx4 acc[2][N];
#pragma unroll
  for (int j = 0; j < N; ++j) acc[0][j] = acc[1][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int groups = static_cast<int>((rb + kGroupBytes - 1) / kGroupBytes);
  const int mine = groups > wv ? (groups - wv + kUpWaves - 1) / kUpWaves : 0;   // groups of this wavefront
  const int turn = static_cast<int>(static_cast<uint32_t>(row0 / kUpRows) * 37u % static_cast<uint32_t>(groups));
  uint32x4 fw[PA][2][2], fx[2][2][N];
  auto place = [&](int i) __attribute__((always_inline)) {   // byte of group i of this wavefront (past the row: none)
    const int q = wv + i * kUpWaves + turn;
    return i < mine ? static_cast<uint32_t>(q < groups ? q : q - groups) * kGroupBytes : rb;
  };
  auto load_w = [&](int p, uint32_t k) __attribute__((always_inline)) {
    w_gate.load(rs_w, k, rb, fw[p][0]);
    w_up.load(rs_w, k, rb, fw[p][1]);
  };
  auto load_x = [&](int p, uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < N; ++j) fx[p][s][j] = load_step(rs_x, ro_x[j], k + s * kStepBytes + g * 16, rb);
  };
#pragma unroll
  for (int p = 0; p < PA; ++p) load_w(p, place(p));
  load_x(0, place(0));
  for (int i = 0; i < mine; i += PA) {
#pragma unroll
    for (int p = 0; p < PA; ++p) {
      load_x((p + 1) % 2, place(i + p + 1));
      uint32x4 sg[2], su[2];
      WeightRows::steps(fw[p][0], sg);
      WeightRows::steps(fw[p][1], su);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          acc[0][j] = mma_step<T>(sg[s], fx[p % 2][s][j], acc[0][j]);
          acc[1][j] = mma_step<T>(su[s], fx[p % 2][s][j], acc[1][j]);
        }
      load_w(p, place(i + p + PA));
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    red[wv][0][j][lane] = acc[0][j];
    red[wv][1][j][lane] = acc[1][j];
  }
  __syncthreads();
  if (wv < N) {
    floatx4 gv = red[0][0][wv][lane], uv = red[0][1][wv][lane];
#pragma unroll
    for (int w = 1; w < kUpWaves; ++w) {
      gv += red[w][0][wv][lane];
      uv += red[w][1][wv][lane];
    }
    // lane 16 g + c: rows 4 g .. 4 g + 3 of column c (f is a multiple of 8, so
    // the four rows exist or none does)
    const int col = 16 * wv + c;
    const int row = row0 + 4 * g;
    if (col < n && row < a.f) {
      const float w = wt[col];
      floatx4 hv;
#pragma unroll
      for (int r = 0; r < 4; ++r) hv[r] = w * (gv[r] / (1.0f + expf(-gv[r])) * uv[r]);
      const int64_t o = static_cast<int64_t>(place0 + col) * a.f + row;
      if constexpr (sizeof(T) == 2) {
        typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
        u16x4 hi, lo;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          hi[r] = to_bf16(hv[r]);
          // an infinite h has no rest (inf - inf would make it NaN)
          const float rest = hv[r] - bf16_to_f32(hi[r]);
          lo[r] = __builtin_fabsf(bf16_to_f32(hi[r])) < __builtin_inff() ? to_bf16(rest) : static_cast<uint16_t>(0);
        }
        uint16_t* h = reinterpret_cast<uint16_t*>(a.h);
        *reinterpret_cast<u16x4*>(h + o) = hi;
        *reinterpret_cast<u16x4*>(h + static_cast<int64_t>(a.T) * a.K * a.f + o) = lo;
      } else {
        *reinterpret_cast<floatx4*>(reinterpret_cast<float*>(a.h) + o) = hv;
      }
    }
  }
}

template <typename T, int N>
__global__ void __launch_bounds__(kUpWaves * kWave) k_moe_up(MoeArgs a) {
  __shared__ Plan pl;
  __shared__ int32_t tok[kMoeTokens];
  __shared__ float wt[kMoeTokens];
  __shared__ floatx4 red[kUpWaves * 2 * N * kWave];
  const int blocks = (a.f + kUpRows - 1) / kUpRows;
  // the tickets of the launch after this one
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.row_blocks; i += kUpWaves * kWave) a.ticket[i] = 0;
  make_plan(a, pl);
  const int i_used = static_cast<int>(blockIdx.x) / blocks;
  if (i_used >= pl.n_used) return;
  const int row0 = (static_cast<int>(blockIdx.x) % blocks) * kUpRows;
  const int e = pl.used[i_used];
  const int n = pl.count[e];
  for (int t = threadIdx.x; t < a.T; t += kUpWaves * kWave) {
    if (!takes(pl, e, t)) continue;
    float w = 0.0f;
    for (int k = 0; k < a.K; ++k)
      if (a.ids[t * a.K + k] == e) w += a.weight[t * a.K + k];
    const int p = place_of(pl, e, t);
    tok[p] = t;
    wt[p] = w;
  }
  __syncthreads();
  const size_t slot_bytes = static_cast<size_t>(3) * a.d * a.f * sizeof(T);
  const __amdgpu_buffer_rsrc_t rs_w = row_buffer(a.slots + pl.slot[e] * slot_bytes, static_cast<uint32_t>(slot_bytes));
  const __amdgpu_buffer_rsrc_t rs_x = row_buffer(a.x, static_cast<uint32_t>(a.T) * a.d * sizeof(T));
  auto pass = [&](auto cols, int p) __attribute__((always_inline)) {
    constexpr int C = decltype(cols)::value;
    up_pass<T, C, C == 1 ? 4 : 2>(a, rs_w, rs_x, row0, tok + p, wt + p, n - p, pl.first[e] + p,
                                  reinterpret_cast<floatx4(*)[2][C][kWave]>(red));
  };
  for (int p = 0; p < n; p += 16 * N) {
    if (p > 0) __syncthreads();   // the last pass's sums are read
    if (N == 1 || n - p <= 16) pass(std::integral_constant<int, 1>(), p);
    else if (N == 2 || n - p <= 32) pass(std::integral_constant<int, N < 2 ? N : 2>(), p);
    else pass(std::integral_constant<int, N>(), p);
  }
}

// ---------------------------------------------------------------- down

// Load groups [m0, m1) of 16 R rows of one expert's Down for up to 16 N of its
// tokens, added to the wavefront's sums own[t][16 R].
template <typename T, int N, int R, int PA>
__device__ __forceinline__ void down_pass(const MoeArgs& a, __amdgpu_buffer_rsrc_t rs_w, __amdgpu_buffer_rsrc_t rs_h,
                                          int row0, int m0, int m1, const uint16_t* tok, int n, int place0, float* own) {
  constexpr int H = sizeof(T) == 2 ? 2 : 1;   // planes of h
  const int lane = threadIdx.x % kWave;
  const int c = lane % 16;
  const int g = lane / 16;
  const uint32_t rb = static_cast<uint32_t>(a.f) * sizeof(T);
  const uint32_t plane = static_cast<uint32_t>(a.T) * a.K * rb;
  uint32_t ro_h[N];
#pragma unroll
  for (int j = 0; j < N; ++j) ro_h[j] = 16 * j + c < n ? static_cast<uint32_t>(place0 + 16 * j + c) * rb : kOutside;
  floatx4 acc[R][N];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < N; ++j) acc[r][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  uint32x4 fw[PA][R][2], fh[2][2][H][N];
  const uint32_t k_end = static_cast<uint32_t>(m1) * kGroupBytes < rb ? static_cast<uint32_t>(m1) * kGroupBytes : rb;
  auto load_w = [&](int p, uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const WeightRows w(row0 + 16 * r, a.d, rb, 0u, c, g);
      w.load(rs_w, k, k_end, fw[p][r]);
    }
  };
  auto load_h = [&](int p, uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int q = 0; q < H; ++q)
          fh[p][s][q][j] = load_step(rs_h, ro_h[j] == kOutside ? kOutside : ro_h[j] + q * plane,
                                     k + s * kStepBytes + g * 16, k_end);
  };
  const uint32_t k0 = static_cast<uint32_t>(m0) * kGroupBytes;
#pragma unroll
  for (int p = 0; p < PA; ++p) load_w(p, k0 + p * kGroupBytes);
  load_h(0, k0);
  for (uint32_t k = k0; k < k_end; k += PA * kGroupBytes) {
#pragma unroll
    for (int p = 0; p < PA; ++p) {
      load_h((p + 1) % 2, k + (p + 1) * kGroupBytes);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        uint32x4 sw[2];
        WeightRows::steps(fw[p][r], sw);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int j = 0; j < N; ++j)
#pragma unroll
            for (int q = 0; q < H; ++q) acc[r][j] = mma_step<T>(sw[s], fh[p % 2][s][q][j], acc[r][j]);
      }
      load_w(p, k + (p + PA) * kGroupBytes);
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (16 * j + c >= n) continue;
    float* o = own + tok[16 * j + c] * (16 * R) + 4 * g;
#pragma unroll
    for (int r = 0; r < R; ++r) *reinterpret_cast<floatx4*>(o + 16 * r) += acc[r][j];
  }
}

// A workgroup owns 16 R output rows and, with splits, one share of the experts'
// products for them: the load groups of all experts in use, one expert after
// the other, are dealt to the splits and to their wavefronts as contiguous
// ranges.  Each wavefront adds its products by token in its own LDS rows; the
// workgroup joins them, and the last of the splits to finish joins theirs.
template <typename T, int N, int R, int NW>
__global__ void __launch_bounds__(NW * kWave) k_moe_down(MoeArgs a) {
  __shared__ Plan pl;
  __shared__ uint16_t tok[kMoeTokens * kMaxK];
  __shared__ int32_t is_last;
  extern __shared__ __align__(16) unsigned char smem[];   // [NW][T][16 R] float32
  float* sums = reinterpret_cast<float*>(smem);
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = tid / kWave;
  const int rbk = static_cast<int>(blockIdx.x) / a.splits;
  const int split = static_cast<int>(blockIdx.x) % a.splits;
  const int row0 = rbk * 16 * R;
  float* own = sums + static_cast<size_t>(wv) * a.T * (16 * R);
  for (int i = lane; i < a.T * 4 * R; i += kWave) reinterpret_cast<floatx4*>(own)[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  make_plan(a, pl);
  for (int i = tid; i < a.T * a.K; i += NW * kWave) {
    const int e = a.ids[i];
    const int t = i / a.K;
    if (e >= 0 && e < a.E && takes(pl, e, t)) tok[pl.first[e] + place_of(pl, e, t)] = static_cast<uint16_t>(t);
  }
  __syncthreads();
  const int groups = (a.f * static_cast<int>(sizeof(T)) + kGroupBytes - 1) / kGroupBytes;   // load groups of a row
  const int64_t total = static_cast<int64_t>(pl.n_used) * groups;
  const int share = split * NW + __builtin_amdgcn_readfirstlane(wv);
  const int shares = a.splits * NW;
  int u = static_cast<int>(total * share / shares);
  const int u1 = static_cast<int>(total * (share + 1) / shares);
  const size_t slot_elems = static_cast<size_t>(3) * a.d * a.f;
  const uint32_t down_bytes = static_cast<uint32_t>(static_cast<size_t>(a.d) * a.f * sizeof(T));
  const uint32_t h_bytes = static_cast<uint32_t>(static_cast<size_t>(a.T) * a.K * a.f * 4);   // two bf16 planes or one float32
  const __amdgpu_buffer_rsrc_t rs_h = row_buffer(a.h, h_bytes);
  while (u < u1) {
    const int i_used = u / groups;
    const int m0 = u - i_used * groups;
    const int m1 = groups - m0 < u1 - u ? groups : m0 + (u1 - u);
    const int e = __builtin_amdgcn_readfirstlane(pl.used[i_used]);
    const int n = __builtin_amdgcn_readfirstlane(pl.count[e]);
    const int first = __builtin_amdgcn_readfirstlane(pl.first[e]);
    const int slot = __builtin_amdgcn_readfirstlane(pl.slot[e]);
    const __amdgpu_buffer_rsrc_t rs_w = row_buffer(
        a.slots + (slot * slot_elems + static_cast<size_t>(2) * a.d * a.f) * sizeof(T), down_bytes);
    auto pass = [&](auto cols, int p) __attribute__((always_inline)) {
      constexpr int C = decltype(cols)::value;
      down_pass<T, C, R, C * R <= 2 ? 4 : 2>(a, rs_w, rs_h, row0, m0, m1, tok + first + p, n - p, first + p, own);
    };
    for (int p = 0; p < n; p += 16 * N) {
      if (N == 1 || n - p <= 16) pass(std::integral_constant<int, 1>(), p);
      else if (N == 2 || n - p <= 32) pass(std::integral_constant<int, N < 2 ? N : 2>(), p);
      else pass(std::integral_constant<int, N>(), p);
    }
    u += m1 - m0;
  }
  __syncthreads();

  // the wavefronts' sums, then the splits', both in order; four rows per thread
  const int quads = a.T * 4 * R;
  if (a.splits > 1) {
    for (int i = tid; i < quads; i += NW * kWave) {
      const int t = i / (4 * R);
      const int row = row0 + 4 * (i % (4 * R));
      if (row >= a.d) continue;
      floatx4 v = reinterpret_cast<floatx4*>(sums)[i];
#pragma unroll
      for (int w = 1; w < NW; ++w) v += reinterpret_cast<floatx4*>(sums)[w * quads + i];
      float* o = a.partial + (static_cast<int64_t>(split) * a.T + t) * a.d + row;
#pragma unroll
      for (int r = 0; r < 4; ++r) __hip_atomic_store(o + r, v[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    wait_vmcnt<0>();
    __syncthreads();
    if (tid == 0)
      is_last = __hip_atomic_fetch_add(&a.ticket[rbk], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                static_cast<uint32_t>(a.splits) - 1u;
    __syncthreads();
    if (!is_last) return;
  }
  for (int i = tid; i < quads; i += NW * kWave) {
    const int t = i / (4 * R);
    const int row = row0 + 4 * (i % (4 * R));
    if (row >= a.d) continue;
    floatx4 v = floatx4{0.f, 0.f, 0.f, 0.f};
    if (a.splits > 1) {
      for (int s = 0; s < a.splits; ++s) {
        const float* o = a.partial + (static_cast<int64_t>(s) * a.T + t) * a.d + row;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += __hip_atomic_load(o + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    } else {
#pragma unroll
      for (int w = 0; w < NW; ++w) v += reinterpret_cast<floatx4*>(sums)[w * quads + i];
    }
    const int64_t o = static_cast<int64_t>(t) * a.d + row;
    if constexpr (sizeof(T) == 2) {
      typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
      u16x4 q = {};
      if (a.residual != nullptr) q = *reinterpret_cast<const u16x4*>(a.residual + o * 2);
#pragma unroll
      for (int r = 0; r < 4; ++r) q[r] = to_bf16(bf16_to_f32(q[r]) + v[r]);
      *reinterpret_cast<u16x4*>(a.out + o * 2) = q;
    } else {
      if (a.residual != nullptr) v = *reinterpret_cast<const floatx4*>(a.residual + o * 4) + v;
      *reinterpret_cast<floatx4*>(a.out + o * 4) = v;
    }
  }
}

// ---------------------------------------------------------------- host

// Rows and wavefronts of k_moe_down's workgroups for launches of T tokens.
struct DownShape {
  int R, NW;
};
DownShape down_shape(int32_t T) { return T <= 16 ? DownShape{1, 16} : (T <= 128 ? DownShape{2, 8} : DownShape{2, 4}); }
int row_blocks_of(int32_t d, int32_t T) { return (d + 16 * down_shape(T).R - 1) / (16 * down_shape(T).R); }
int splits_of(int32_t d, int32_t T) {
  const int blocks = row_blocks_of(d, T);
  const int want = 4096 / down_shape(T).NW;   // workgroups that fill the GPU: 16 wavefronts per CU
  const int s = (want + blocks - 1) / blocks;
  return s < kMaxSplits ? s : kMaxSplits;
}

template <typename T, int N, int R, int NW>
hipError_t launch(MoeArgs a, hipStream_t st) {
  const int experts = a.E < a.T * a.K ? a.E : a.T * a.K;   // at most this many are in use
  const unsigned up = static_cast<unsigned>(experts) * static_cast<unsigned>((a.f + kUpRows - 1) / kUpRows);
  k_moe_up<T, N><<<up, kUpWaves * kWave, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto kern = k_moe_down<T, N, R, NW>;
  const size_t lds = static_cast<size_t>(NW) * a.T * 16 * R * sizeof(float);
  if (lds + 16384 > 65536) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                            static_cast<int>(lds));
    if (e != hipSuccess) return e;
  }
  kern<<<static_cast<unsigned>(a.row_blocks) * static_cast<unsigned>(a.splits), NW * kWave, lds, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t experts(const MoeArgs& a, hipStream_t st) {   // as down_shape
  if (a.T <= 16) return launch<T, 1, 1, 16>(a, st);
  if (a.T <= 32) return launch<T, 2, 2, 8>(a, st);
  if (a.T <= 128) return launch<T, 4, 2, 8>(a, st);
  return launch<T, 4, 2, 4>(a, st);
}

// Workspace of one launch: [h][partial sums][tickets], each 256-byte aligned; a
// launch of fewer tokens never needs more.
size_t parts(int32_t d, int32_t f, int32_t T, int32_t K, size_t* partial, size_t* ticket) {
  size_t o = align_up(static_cast<size_t>(T) * K * f * 4, kAlign);
  *partial = o;
  o += align_up(static_cast<size_t>(splits_of(d, T)) * T * d * sizeof(float), kAlign);
  *ticket = o;
  return o + align_up(static_cast<size_t>((d + 15) / 16) * sizeof(uint32_t), kAlign);   // (the most row blocks of any T)
}

}  // namespace

size_t moe_workspace_bytes(int32_t d, int32_t f, fm_dtype, int32_t T, int32_t K) {
  size_t p, k;
  return parts(d, f, T < kMoeTokens ? T : kMoeTokens, K, &p, &k);
}

hipError_t launch_moe_experts(const fm_expert_cache& c, const void* x, const int32_t* ids, const float* weight,
                              int32_t T, int32_t K, const void* residual, void* out, uint32_t* flags, void* ws,
                              hipStream_t st) {
  const size_t es = c.dtype == FM_BF16 ? 2 : 4;
  const size_t row = static_cast<size_t>(c.d) * es;
  for (int32_t t0 = 0; t0 < T; t0 += kMoeTokens) {
    MoeArgs a;
    a.T = T - t0 < kMoeTokens ? T - t0 : kMoeTokens;
    size_t partial, ticket;
    parts(c.d, c.f, a.T, K, &partial, &ticket);
    a.slots = static_cast<const char*>(c.slots);
    a.slot_of = c.slot_of;
    a.x = static_cast<const char*>(x) + t0 * row;
    a.ids = ids + static_cast<int64_t>(t0) * K;
    a.weight = weight + static_cast<int64_t>(t0) * K;
    a.residual = residual == nullptr ? nullptr : static_cast<const char*>(residual) + t0 * row;
    a.out = static_cast<char*>(out) + t0 * row;
    a.h = static_cast<char*>(ws);
    a.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + partial);
    a.ticket = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + ticket);
    a.flags = flags;
    a.K = K;
    a.E = c.E;
    a.n_slots = c.n_slots;
    a.d = c.d;
    a.f = c.f;
    a.splits = splits_of(c.d, a.T);
    a.row_blocks = row_blocks_of(c.d, a.T);
    const hipError_t e = c.dtype == FM_BF16 ? experts<uint16_t>(a, st) : experts<float>(a, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fm
