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
constexpr int kUpRows = 16;        // rows of Gate and of Up per block
constexpr int kMaxSplits = 16;     // workgroups that share one block of output rows
constexpr int kGroupBytes = 2 * kStepBytes;   // of every row in one load group
constexpr int kMaxTiles = 4;       // tiles of 16 tokens in one pass over an expert's weights

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

// Which tokens take which experts, in LDS, for launches of up to MAXT tokens.
// An expert's tokens, in order, are its places; the experts' places follow each
// other.  An entry is one pass over an expert's weights for up to 64 of its
// places; entries are ordered by their tiles of 16 (1, 2 or 4).
template <int MAXT>
struct Plan {
  static constexpr int kWords = (MAXT + 63) / 64;
  static constexpr int kPairs = MAXT * kMaxK;
  static constexpr int kEntries = kMaxE + kPairs / 64;
  uint64_t takes[kMaxE][kWords];   // tokens that take the expert
  int32_t slot[kMaxE];
  int32_t entry_slot[kEntries];
  uint16_t entry_place[kEntries];  // the entry's first place
  uint16_t entry_n[kEntries];      // and its places
  int32_t classes[3];              // ends of the entries of 1, 2 and 4 tiles
  uint16_t tok[kPairs];            // token of each place
  float weight[kPairs];            // and its weight
  int32_t again;                   // some token lists an expert twice
};

// Filled by the whole workgroup; ends with a barrier.
template <int MAXT, int NT>
__device__ __forceinline__ void make_plan(const MoeArgs& a, Plan<MAXT>& pl) {
  using P = Plan<MAXT>;
  constexpr int kOwn = (P::kPairs + NT - 1) / NT;
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int pairs = a.T * a.K;
  // every load before the first barrier
  int id[kOwn];
  float wt[kOwn];
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    id[j] = tid + j * NT < pairs ? a.ids[tid + j * NT] : -1;
    wt[j] = tid + j * NT < pairs ? a.weight[tid + j * NT] : 0.0f;
  }
  if (tid == 0) pl.again = 0;
  if (tid < kMaxE) pl.slot[tid] = tid < a.E ? a.slot_of[tid] : -1;
  for (int i = tid; i < kMaxE * P::kWords; i += NT) pl.takes[i / P::kWords][i % P::kWords] = 0;
  __syncthreads();
  uint32_t bad = 0;
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    if (id[j] < 0) continue;
    const int s = id[j] < a.E ? pl.slot[id[j]] : 0;
    if (id[j] >= a.E || s >= a.n_slots) {
      bad |= FM_FLAG_INDEX_RANGE;
      id[j] = -1;
    } else if (s < 0) {
      bad |= FM_FLAG_EXPERT_MISSING;
      id[j] = -1;
    } else {
      const int t = (tid + j * NT) / a.K;
      const uint64_t bit = 1ull << (t % 64);
      if ((atomicOr(reinterpret_cast<unsigned long long*>(&pl.takes[id[j]][t / 64]), bit) & bit) != 0) pl.again = 1;
    }
  }
  if (bad != 0 && a.flags != nullptr && blockIdx.x == 0) atomicOr(a.flags, bad);
  __syncthreads();
  // each wavefront counts for itself, an expert per lane; the first writes the entries
  int n = 0;
#pragma unroll
  for (int j = 0; j < P::kWords; ++j) n += __popcll(pl.takes[lane][j]);
  auto scan = [&](int v) {   // exclusive, over the lanes
    int incl = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int u = __shfl_up(incl, o, kWave);
      if (lane >= o) incl += u;
    }
    return incl - v;
  };
  const int first = scan(n);
  if (tid < kWave) {
    const int rest = n % 64;
    const int in1 = rest > 0 && rest <= 16 ? 1 : 0;
    const int in2 = rest > 16 && rest <= 32 ? 1 : 0;
    const int in4 = n / 64 + (rest > 32 ? 1 : 0);
    const int n1 = __popcll(__ballot(in1 != 0));
    const int n2 = __popcll(__ballot(in2 != 0));
    const uint64_t below = (1ull << lane) - 1ull;
    auto put = [&](int i, int place, int count) {
      pl.entry_slot[i] = pl.slot[lane];
      pl.entry_place[i] = static_cast<uint16_t>(place);
      pl.entry_n[i] = static_cast<uint16_t>(count);
    };
    const uint64_t m1 = __ballot(in1 != 0), m2 = __ballot(in2 != 0);
    if (in1) put(__popcll(m1 & below), first + n - rest, rest);
    if (in2) put(n1 + __popcll(m2 & below), first + n - rest, rest);
    int n4 = 0;
    if constexpr (MAXT > 32) {
      const int p4 = scan(in4);
      for (int j = 0; j < in4; ++j) put(n1 + n2 + p4 + j, first + 64 * j, n - 64 * j < 64 ? n - 64 * j : 64);
      n4 = __shfl(p4 + in4, kWave - 1, kWave);
    }
    if (lane == 0) {
      pl.classes[0] = n1;
      pl.classes[1] = n1 + n2;
      pl.classes[2] = n1 + n2 + n4;
    }
  }
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int e = id[j];
    const int base = __shfl(first, e < 0 ? 0 : e, kWave);
    if (e < 0) continue;
    const int t = (tid + j * NT) / a.K;
    int p = base + __popcll(pl.takes[e][t / 64] & ((1ull << (t % 64)) - 1ull));
    for (int q = 0; q < t / 64; ++q) p += __popcll(pl.takes[e][q]);
    // an expert that the token lists again counts with both weights (every
    // listing writes the same place and sum)
    float w = wt[j];
    if (pl.again != 0) {
      w = 0.0f;
      for (int k = 0; k < a.K; ++k)
        if (a.ids[t * a.K + k] == e) w += a.weight[t * a.K + k];
    }
    pl.tok[p] = static_cast<uint16_t>(t);
    pl.weight[p] = w;
  }
  __syncthreads();
}

__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }

// Load groups of R tiles of 16 weight rows and of C tiles of 16 activation
// columns in H planes, PA groups in flight.  Loads finish in the order of their
// issue, so both operands of a group go out together: an activation issued after
// the weights of later groups would wait for them.
template <typename T, int C, int R, int H, int PA>
struct Stream {
  uint32x4 w[PA][R][2], b[PA][H][C][2];
  __device__ __forceinline__ void load(int p, __amdgpu_buffer_rsrc_t rs_w, const RowPairs (&rows)[R],
                                       __amdgpu_buffer_rsrc_t rs_b, const RowPairs (&cols)[C], uint32_t plane,
                                       uint32_t k, uint32_t k_end) {
#pragma unroll
    for (int r = 0; r < R; ++r) rows[r].template load<kStream>(rs_w, k, k_end, w[p][r]);
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int q = 0; q < H; ++q) {
        RowPairs c = cols[j];
        if (q > 0) {
          if (c.even != kOutside) c.even += plane;
          if (c.odd != kOutside) c.odd += plane;
        }
        c.template load<kKeep>(rs_b, k, k_end, b[p][q][j]);
      }
  }
  __device__ __forceinline__ void multiply(int p, floatx4 (&acc)[R][C]) const {
    uint32x4 sw[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r) RowPairs::steps(w[p][r], sw[r]);
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int q = 0; q < H; ++q) {
        uint32x4 sb[2];
        RowPairs::steps(b[p][q][j], sb);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int r = 0; r < R; ++r) acc[r][j] = mma_step<T>(sw[r][s], sb[s], acc[r][j]);
      }
  }
};

template <int R, int C>
__device__ __forceinline__ void clear(floatx4 (&acc)[R][C]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < C; ++j) acc[r][j] = floatx4{0.f, 0.f, 0.f, 0.f};
}

// ---------------------------------------------------------------- gate and up

// The workgroup's units (a block of 16 gate and 16 up rows of one entry) among
// the entries e0 .. e1 - 1, all of C tiles: every gridDim.x-th unit of the
// concatenated entries.  The wavefronts deal the load groups of a row among
// themselves, starting at a place that differs from block to block: rows of a
// power of two bytes would otherwise keep all workgroups on few memory channels
// at a time (2 GB in rows of 8 KB: 5.9 -> 7.1 TB/s).  The loads of a unit's first
// groups go out before the last unit's products are done.
template <typename T, int MAXT, int C, int PA>
__device__ __forceinline__ void up_units(const MoeArgs& a, const Plan<MAXT>& pl, int e0, int e1,
                                         floatx4 (*red)[C][kWave]) {
  const int lane = threadIdx.x % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane % 16;
  const int g = lane / 16;
  const uint32_t rb = static_cast<uint32_t>(a.d) * sizeof(T);
  const int groups = static_cast<int>((rb + kGroupBytes - 1) / kGroupBytes);
  const int mine = groups > wv ? (groups - wv + kUpWaves - 1) / kUpWaves : 0;   // groups of this wavefront
  const int rounds = ((groups + kUpWaves - 1) / kUpWaves + PA - 1) / PA;        // of PA groups, for every wavefront
  const int blocks = (a.f + kUpRows - 1) / kUpRows;
  const int grid = static_cast<int>(gridDim.x);
  const int u_end = e1 * blocks;
  int u = e0 * blocks;
  u += (static_cast<int>(blockIdx.x) - u % grid + grid) % grid;
  if (u >= u_end) return;
  const size_t slot_bytes = static_cast<size_t>(3) * a.d * a.f * sizeof(T);
  const __amdgpu_buffer_rsrc_t rs_x = row_buffer(a.x, static_cast<uint32_t>(a.T) * rb);
  // the unit that is being loaded
  __amdgpu_buffer_rsrc_t rs_w = rs_x;
  RowPairs rows[2] = {}, cols[C] = {};
  int turn = 0;
  uint32_t k_end = 0;
  auto aim = [&](int v) __attribute__((always_inline)) {
    if (v >= u_end) {
      k_end = 0;   // nothing more to load
      return;
    }
    k_end = rb;
    const int e = v / blocks;
    const int blk = v - e * blocks;
    rs_w = row_buffer(a.slots + __builtin_amdgcn_readfirstlane(pl.entry_slot[e]) * slot_bytes,
                      static_cast<uint32_t>(slot_bytes));
    rows[0] = RowPairs(blk * kUpRows, a.f, rb, 0u);
    rows[1] = RowPairs(blk * kUpRows, a.f, rb, static_cast<uint32_t>(a.f) * rb);
    const int n = pl.entry_n[e], p0 = pl.entry_place[e];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int q = 16 * j + c / 2 * 2;
      cols[j].even = q < n ? static_cast<uint32_t>(pl.tok[p0 + q]) * rb + RowPairs::place() : kOutside;
      cols[j].odd = q + 1 < n ? static_cast<uint32_t>(pl.tok[p0 + q + 1]) * rb + RowPairs::place() : kOutside;
    }
    turn = static_cast<int>(static_cast<uint32_t>(blk) * 37u % static_cast<uint32_t>(groups));
  };
  Stream<T, C, 2, 1, PA> st;
  auto load = [&](int p, int i) __attribute__((always_inline)) {   // the wavefront's i-th group
    const int q = wv + i * kUpWaves + turn;
    st.load(p, rs_w, rows, rs_x, cols, 0u, static_cast<uint32_t>(q < groups ? q : q - groups) * kGroupBytes,
            i < mine ? k_end : 0u);
  };
  aim(u);
#pragma unroll
  for (int p = 0; p < PA; ++p) load(p, p);
  for (; u < u_end; u += grid) {
    floatx4 acc[2][C];
    clear(acc);
    for (int r = 0; r < rounds; ++r) {
      const bool next = r + 1 == rounds;
      if (next) aim(u + grid);
#pragma unroll
      for (int p = 0; p < PA; ++p) {
        st.multiply(p, acc);
        load(p, next ? p : (r + 1) * PA + p);
      }
    }
    // the wavefronts' sums meet in LDS, gate's and then up's
    floatx4 sum[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      wait_lgkm0();
      raw_barrier();   // the sums before are read
#pragma unroll
      for (int j = 0; j < C; ++j) red[wv][j][lane] = acc[m][j];
      wait_lgkm0();
      raw_barrier();
      if (wv < C) {
        sum[m] = red[0][wv][lane];
#pragma unroll
        for (int w = 1; w < kUpWaves; ++w) sum[m] += red[w][wv][lane];
      }
    }
    if (wv >= C) continue;
    const floatx4 gv = sum[0], uv = sum[1];
    // lane 16 g + c: rows 4 g .. 4 g + 3 of column c (f is a multiple of 8, so
    // the four rows exist or none does)
    const int e = u / blocks;
    const int col = 16 * wv + c;
    const int row = (u - e * blocks) * kUpRows + 4 * g;
    if (col >= pl.entry_n[e] || row >= a.f) continue;
    const int place = pl.entry_place[e] + col;
    const float w = pl.weight[place];
    floatx4 hv;
#pragma unroll
    for (int r = 0; r < 4; ++r) hv[r] = w * (gv[r] / (1.0f + expf(-gv[r])) * uv[r]);
    const int64_t o = static_cast<int64_t>(place) * a.f + row;
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
  wait_lgkm0();
}

// Tokens of a launch of N tiles: up to 16 N, or any number for N = 4.
constexpr int max_tokens(int N) { return N < kMaxTiles ? 16 * N : kMoeTokens; }

template <typename T, int N>
__global__ void __launch_bounds__(kUpWaves * kWave, N == 1 ? 4 : 2) k_moe_up(MoeArgs a) {
  constexpr int MAXT = max_tokens(N);
  __shared__ Plan<MAXT> pl;
  __shared__ floatx4 red[kUpWaves * N * kWave];
  // the tickets of the launch after this one
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.row_blocks; i += kUpWaves * kWave) a.ticket[i] = 0;
  make_plan<MAXT, kUpWaves * kWave>(a, pl);
  auto run = [&](auto tiles, auto depth, int e0, int e1) __attribute__((always_inline)) {
    constexpr int C = decltype(tiles)::value;
    if (e0 < e1)
      up_units<T, MAXT, C, decltype(depth)::value>(a, pl, e0, e1, reinterpret_cast<floatx4(*)[C][kWave]>(red));
  };
  run(std::integral_constant<int, 1>(), std::integral_constant<int, N == 1 ? 2 : 4>(), 0, pl.classes[0]);
  if constexpr (N >= 2) run(std::integral_constant<int, 2>(), std::integral_constant<int, 4>(), pl.classes[0], pl.classes[1]);
  if constexpr (N == 4) run(std::integral_constant<int, 4>(), std::integral_constant<int, 2>(), pl.classes[1], pl.classes[2]);
}

// ---------------------------------------------------------------- down

// Load groups [u, u1) of the concatenated entries, those among entries e0 .. e1 - 1
// (all of C tiles), for 16 R output rows; an entry's products are added to the
// wavefront's sums own[t][16 R].
template <typename T, int MAXT, int C, int R, int NW, int PA>
__device__ __forceinline__ void down_groups(const MoeArgs& a, const Plan<MAXT>& pl, int e0, int e1, int row0, int groups,
                                            int64_t share_u0, int64_t share_u1, int wv, float* own) {
  constexpr int H = sizeof(T) == 2 ? 2 : 1;   // planes of h
  const int lane = threadIdx.x % kWave;
  const int c = lane % 16;
  const int g = lane / 16;
  const uint32_t rb = static_cast<uint32_t>(a.f) * sizeof(T);
  const uint32_t plane = static_cast<uint32_t>(a.T) * a.K * rb;
  int u = static_cast<int>(share_u0 > static_cast<int64_t>(e0) * groups ? share_u0 : static_cast<int64_t>(e0) * groups);
  const int u1 = static_cast<int>(share_u1 < static_cast<int64_t>(e1) * groups ? share_u1 : static_cast<int64_t>(e1) * groups);
  if (u >= u1) return;
  const size_t slot_elems = static_cast<size_t>(3) * a.d * a.f;
  const uint32_t down_bytes = static_cast<uint32_t>(static_cast<size_t>(a.d) * a.f * sizeof(T));
  const __amdgpu_buffer_rsrc_t rs_h =
      row_buffer(a.h, static_cast<uint32_t>(static_cast<size_t>(a.T) * a.K * a.f * 4));   // two bf16 planes or one float32
  RowPairs rows[R], cols[C] = {};
#pragma unroll
  for (int r = 0; r < R; ++r) rows[r] = RowPairs(row0 + 16 * r, a.d, rb, 0u);
  // the entry that is being loaded: this wavefront's groups k, k + NW, ... of it
  __amdgpu_buffer_rsrc_t rs_w = rs_h;
  uint32_t k = 0, k_end = 0;
  int l = u;
  const int u_first = u;
  auto aim = [&]() __attribute__((always_inline)) {
    if (l >= u1) {
      k = k_end = 0;
      return;
    }
    const int e = l / groups;
    const int m0 = l - e * groups;
    const int m1 = groups - m0 < u1 - l ? groups : m0 + (u1 - l);
    rs_w = row_buffer(a.slots + (__builtin_amdgcn_readfirstlane(pl.entry_slot[e]) * slot_elems +
                                 static_cast<size_t>(2) * a.d * a.f) * sizeof(T), down_bytes);
    const int n = pl.entry_n[e], p0 = pl.entry_place[e];
#pragma unroll
    for (int j = 0; j < C; ++j) cols[j] = RowPairs(16 * j, n, rb, static_cast<uint32_t>(p0) * rb);
    // (dealt on from where the last entry's groups ended)
    k = static_cast<uint32_t>(m0 + (wv + NW - (l - u_first) % NW) % NW) * kGroupBytes;
    k_end = static_cast<uint32_t>(m1) * kGroupBytes < rb ? static_cast<uint32_t>(m1) * kGroupBytes : rb;
    l += m1 - m0;
  };
  Stream<T, C, R, H, PA> st;
  aim();
#pragma unroll
  for (int p = 0; p < PA; ++p) st.load(p, rs_w, rows, rs_h, cols, plane, k + p * NW * kGroupBytes, k_end);
  while (u < u1) {
    const int e = u / groups;
    const int m0 = u - e * groups;
    const int m = groups - m0 < u1 - u ? groups - m0 : u1 - u;   // groups of this entry
    floatx4 acc[R][C];
    clear(acc);
    for (int i = 0; i < m; i += PA * NW) {
      k += PA * NW * kGroupBytes;
      if (i + PA * NW >= m) aim();
#pragma unroll
      for (int p = 0; p < PA; ++p) {
        st.multiply(p, acc);
        st.load(p, rs_w, rows, rs_h, cols, plane, k + p * NW * kGroupBytes, k_end);
      }
    }
    const int n = pl.entry_n[e], p0 = pl.entry_place[e];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if (16 * j + c >= n) continue;
      float* o = own + pl.tok[p0 + 16 * j + c] * (16 * R) + 4 * g;
#pragma unroll
      for (int r = 0; r < R; ++r) *reinterpret_cast<floatx4*>(o + 16 * r) += acc[r][j];
    }
    u += m;
  }
}

// A workgroup owns 16 R output rows and, with splits, one share of the experts'
// products for them: the load groups of all entries, one entry after the other,
// are dealt to the splits and to their wavefronts as contiguous ranges.  Each
// wavefront adds its products by token in its own LDS rows; the workgroup joins
// them, and the last of the splits to finish joins theirs.
template <typename T, int N, int R, int NW>
__global__ void __launch_bounds__(NW * kWave, N == 4 ? 2 : 4) k_moe_down(MoeArgs a) {
  constexpr int MAXT = max_tokens(N);
  __shared__ Plan<MAXT> pl;
  __shared__ int32_t is_last;
  extern __shared__ __align__(16) unsigned char smem[];   // [NW][T][16 R] float32
  float* sums = reinterpret_cast<float*>(smem);
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int rbk = static_cast<int>(blockIdx.x) / a.splits;
  const int split = static_cast<int>(blockIdx.x) % a.splits;
  const int row0 = rbk * 16 * R;
  float* own = sums + static_cast<size_t>(wv) * a.T * (16 * R);
  for (int i = lane; i < a.T * 4 * R; i += kWave) reinterpret_cast<floatx4*>(own)[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  make_plan<MAXT, NW * kWave>(a, pl);
  const int groups = (a.f * static_cast<int>(sizeof(T)) + kGroupBytes - 1) / kGroupBytes;   // load groups of a row
  const int64_t total = static_cast<int64_t>(pl.classes[2]) * groups;
  const int64_t u0 = total * split / a.splits;
  const int64_t u1 = total * (split + 1) / a.splits;
  auto run = [&](auto tiles, auto depth, int e0, int e1) __attribute__((always_inline)) {
    if (e0 < e1)
      down_groups<T, MAXT, decltype(tiles)::value, R, NW, decltype(depth)::value>(a, pl, e0, e1, row0, groups, u0, u1, wv, own);
  };
  run(std::integral_constant<int, 1>(), std::integral_constant<int, N == 4 ? 4 : 2>(), 0, pl.classes[0]);
  if constexpr (N >= 2)
    run(std::integral_constant<int, 2>(), std::integral_constant<int, N == 4 ? 3 : 2>(), pl.classes[0], pl.classes[1]);
  if constexpr (N == 4) run(std::integral_constant<int, 4>(), std::integral_constant<int, 2>(), pl.classes[1], pl.classes[2]);
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
DownShape down_shape(int32_t T) { return T <= 128 ? DownShape{2, 8} : DownShape{2, 4}; }
int row_blocks_of(int32_t d, int32_t T) { return (d + 16 * down_shape(T).R - 1) / (16 * down_shape(T).R); }
int splits_of(int32_t d, int32_t T) {
  const int blocks = row_blocks_of(d, T);
  const int want = 4096 / down_shape(T).NW;   // workgroups that fill the GPU: 16 wavefronts per CU
  const int s = (want + blocks - 1) / blocks;
  return s < kMaxSplits ? s : kMaxSplits;
}

constexpr int kCus = 256;

template <typename T, int N, int R, int NW>
hipError_t launch(MoeArgs a, hipStream_t st) {
  // at most this many units; each workgroup takes its turn at them
  const int experts = a.E + a.T * a.K / 64 < a.T * a.K ? a.E + a.T * a.K / 64 : a.T * a.K;
  const int units = experts * ((a.f + kUpRows - 1) / kUpRows);
  const int fill = N == 1 ? 2 * kCus : kCus;
  k_moe_up<T, N><<<static_cast<unsigned>(units < fill ? units : fill), kUpWaves * kWave, 0, st>>>(a);
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
  if (a.T <= 16) return launch<T, 1, 2, 8>(a, st);
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
