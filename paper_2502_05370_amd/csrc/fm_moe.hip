// The chosen experts' products of one MoE layer, on experts that sit in the slots
// of an expert cache: for the few tokens of a decode iteration, and for prompts.
//
//   h[t,e]  = weight(t,e) * silu(Gate_e x[t]) * (Up_e x[t])
//   out[t]  = residual[t] + sum over e of Down_e h[t,e]
//
// With few tokens each weight meets a handful of columns, so reading every
// expert in use once from HBM bounds both products (6 T K d f operations on
// 6 d f bytes per expert in bf16; one with more than 64 of up to 128 tokens is
// read once per 64).  Weights go straight from memory to the
// registers of the matrix instructions, 16 rows by 128 contiguous bytes per load
// group.  Up to 16 tokens two launches, k_moe_up (Gate and Up, joined to h) and
// k_moe_down: the wavefronts of a workgroup split the long axis, which keeps many
// loads in flight for any number of experts, their sums meet in LDS in a fixed
// order, and the activations come from the caches.  More tokens take three
// (k_moe_up_rows, k_moe_down_rows, k_moe_join): the wavefronts own weight rows and
// share the activations through LDS.  Above 128 the matrix instructions come to
// bound them, and four launches (k_moe_list, k_moe_up_long, k_moe_down_long,
// k_moe_sum) take up to 4,096 tokens.
//
// Measured, one MI355X, bf16: 8 tokens through 16 experts of 4,096 x 6,400 (1.65
// GB of weights in use) 162 + 89 us, 6.6 TB/s; 64 tokens through 8 of 4,096 x
// 14,336 (2.82 GB) 330 + 146 + 5 us, 5.9 TB/s; one token through 4 of 60 of
// 2,048 x 1,408 (69 MB) 15 + 13 us, of which reading takes 10: the plan, the first
// loads' latency and the joins of two dependent launches are the rest; 2,048 tokens
// through 16 of 4,096 x 6,400, two each, 8 + 595 + 490 + 18 us, 584 TFLOP/s.
//
// h keeps 16 bits of mantissa in bf16 models: it is stored as the bf16 below it (in
// magnitude) and the nearest bf16 of the rest, 2^-16 of h at most from it, both
// multiplied, so that the only rounding to bf16 that shows is the output's own.  With few tokens the weights' stream
// bounds the second product, and the extra matrix instructions hide behind it; in
// long batches they are a quarter of all, the price of results that do not depend
// on the batch's length by more than sums' order.
#include "fm_internal.h"
#include "fm_mma.h"

namespace fm {

namespace {

constexpr int kUpWaves = 8;
constexpr int kUpRows = 16;        // rows of Gate and of Up per block
constexpr int kDownWaves = 8;
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
  // unit u of n entries of `blocks` row blocks each
  __device__ __forceinline__ int token(int place) const { return tok[place]; }
  __device__ __forceinline__ float weight_of(int place) const { return weight[place]; }
  static __device__ __forceinline__ int entry(int u, int blocks, int) { return u / blocks; }
  static __device__ __forceinline__ int block(int u, int blocks, int) { return u % blocks; }
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
// columns in H planes, PA groups in flight (a third one, on more registers, costs
// as much as it hides).  Loads finish in the order of their
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

constexpr uint16_t kNanBf16 = 0x7FC0;
constexpr float kLeast = 0x1p-126f;   // the least normal bf16 (and float32)

// Four rows of h of one place.
template <typename T>
__device__ __forceinline__ void store_h(const MoeArgs& a, int place, int row, floatx4 hv) {
  const int64_t o = static_cast<int64_t>(place) * a.f + row;
  if constexpr (sizeof(T) == 2) {
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    u16x4 hi, lo;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      // towards zero: a finite h beyond the largest bf16 stays finite
      hi[r] = hv[r] == hv[r] ? static_cast<uint16_t>(__float_as_uint(hv[r]) >> 16) : kNanBf16;
      // The rest has h's sign and is zero only if h is, so that its product with an
      // infinite weight is the first one's infinity, no NaN.  Where nothing is left
      // (or h is infinite) 2^-126 stands for it, below a float32's normal range.
      const float rest = hv[r] - bf16_to_f32(hi[r]);
      const float least = hv[r] == 0.0f ? 0.0f : __builtin_copysignf(kLeast, hv[r]);
      lo[r] = to_bf16(__builtin_fabsf(rest) >= kLeast ? rest : least);
    }
    uint16_t* h = reinterpret_cast<uint16_t*>(a.h);
    *reinterpret_cast<u16x4*>(h + o) = hi;
    *reinterpret_cast<u16x4*>(h + static_cast<int64_t>(a.T) * a.K * a.f + o) = lo;
  } else {
    *reinterpret_cast<floatx4*>(reinterpret_cast<float*>(a.h) + o) = hv;
  }
}

// Four outputs: the residual and the sums.
template <typename T>
__device__ __forceinline__ void store_out(const MoeArgs& a, int64_t o, floatx4 v) {
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
    store_h<T>(a, place, row, hv);
  }
  wait_lgkm0();
}

template <typename T>
__global__ void __launch_bounds__(kUpWaves * kWave, 4) k_moe_up(MoeArgs a) {
  __shared__ Plan<16> pl;
  __shared__ floatx4 red[kUpWaves][1][kWave];
  // the tickets of the launch after this one
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.row_blocks; i += kUpWaves * kWave) a.ticket[i] = 0;
  make_plan<16, kUpWaves * kWave>(a, pl);
  up_units<T, 16, 1, 2>(a, pl, 0, pl.classes[2], red);
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
template <typename T>
__global__ void __launch_bounds__(kDownWaves * kWave, 4) k_moe_down(MoeArgs a) {
  constexpr int R = 2, NW = kDownWaves;
  __shared__ Plan<16> pl;
  __shared__ int32_t is_last;
  __shared__ floatx4 smem[NW * 16 * 4 * R];   // [NW][T][16 R] float32
  float* sums = reinterpret_cast<float*>(smem);
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int rbk = static_cast<int>(blockIdx.x) / a.splits;
  const int split = static_cast<int>(blockIdx.x) % a.splits;
  const int row0 = rbk * 16 * R;
  float* own = sums + static_cast<size_t>(wv) * a.T * (16 * R);
  for (int i = lane; i < a.T * 4 * R; i += kWave) reinterpret_cast<floatx4*>(own)[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  make_plan<16, NW * kWave>(a, pl);
  const int groups = (a.f * static_cast<int>(sizeof(T)) + kGroupBytes - 1) / kGroupBytes;   // load groups of a row
  const int64_t total = static_cast<int64_t>(pl.classes[2]) * groups;
  const int64_t u0 = total * split / a.splits;
  const int64_t u1 = total * (split + 1) / a.splits;
  down_groups<T, 16, 1, R, NW, 2>(a, pl, 0, pl.classes[2], row0, groups, u0, u1, wv, own);
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
    store_out<T>(a, static_cast<int64_t>(t) * a.d + row, v);
  }
}

// ---------------------------------------------------------------- more tokens

// From 17 tokens on a workgroup's eight wavefronts own different weight rows and
// share the activations: with up to 64 columns those would otherwise be read from
// the L2 as often as the weights from HBM, and a CU's loads cannot serve both
// (64 tokens through 8 experts of 4,096 x 14,336: 535 us that way, 480 this).
// They pass through LDS a slab of SG load groups at a time, two slabs deep; the
// weights keep going straight to registers, a slab ahead.
constexpr int kRowWaves = 8;

// One slab of the sequence that a workgroup streams.
template <int C, int H, int R>
struct Slab {
  __amdgpu_buffer_rsrc_t w;
  RowPairs rows[R];
  uint32_t col[H][C];     // where the columns that this thread copies start
  uint32_t k, k_end;      // bytes of the rows; zeros from k_end on
  bool last;              // of its unit or entry
};

// next(slab) sets the slab after the one it set last (false: none left);
// done(acc) takes the sums after a slab that is the last.  Called by the whole
// workgroup; buf holds two slabs of columns.
template <typename T, int C, int H, int R, int SG, typename Next, typename Done>
__device__ __forceinline__ void stream_slabs(__amdgpu_buffer_rsrc_t rs_b, unsigned char* buf, Next next, Done done) {
  constexpr int kChunks = SG * 8;                       // 16-byte pieces of a column in a slab
  constexpr int kCol = SG * RowPairs::kBytes + 16;      // (the odd piece keeps the columns' banks apart)
  constexpr int kSlab = H * C * 16 * kCol;
  static_assert(kRowWaves * kWave == 16 * kChunks || kRowWaves * kWave == 32 * kChunks, "threads per column piece");
  constexpr int kCols = kRowWaves * kWave / kChunks;    // columns per pass of the threads
  constexpr int NB = H * C * 16 / kCols;                // pieces of each thread
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int c = lane % 16;
  const int g = lane / 16;
  uint32x4 piece[NB];
  uint32x4 fw[SG][R][2];
  floatx4 acc[R][C];
  Slab<C, H, R> slab;   // that is being loaded
  auto load_b = [&]() __attribute__((always_inline)) {
    const uint32_t at = static_cast<uint32_t>(tid % kChunks) * 16u;
    const bool in = slab.k + at < slab.k_end;
    const int ks = static_cast<int>(slab.k < slab.k_end ? slab.k : 0u);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const uint32_t col = slab.col[i / (NB / H)][i % (NB / H)];
      piece[i] = __builtin_amdgcn_raw_buffer_load_b128(
          rs_b, static_cast<int>(in && col != kOutside ? col + at : kOutside), ks, kKeep);
    }
  };
  auto store_b = [&](unsigned char* to) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
      *reinterpret_cast<uint32x4*>(to + (i * kCols + tid / kChunks) * kCol + tid % kChunks * 16) = piece[i];
  };
  auto load_w = [&](int p) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      slab.rows[r].template load<kStream>(slab.w, slab.k + p * RowPairs::kBytes, slab.k_end, fw[p][r]);
  };
  raw_barrier();   // the buffers are free
  if (!next(slab)) return;
  load_b();
#pragma unroll
  for (int p = 0; p < SG; ++p) load_w(p);
  store_b(buf);
  wait_lgkm0();
  raw_barrier();
  clear(acc);
  for (int turn = 0;; turn ^= 1) {
    const bool last = slab.last;
    const bool more = next(slab);
    if (!more) slab.k = slab.k_end = 0;   // (its buffer stands)
    load_b();
    const unsigned char* from = buf + turn * kSlab;
#pragma unroll
    for (int p = 0; p < SG; ++p) {
      uint32x4 sw[R][2];
#pragma unroll
      for (int r = 0; r < R; ++r) RowPairs::steps(fw[p][r], sw[r]);
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int q = 0; q < H; ++q)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const uint32x4 b = *reinterpret_cast<const uint32x4*>(
                from + (q * C * 16 + 16 * j + c) * kCol + p * RowPairs::kBytes + 32 * g + 16 * s);
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r][j] = mma_step<T>(sw[r][s], b, acc[r][j]);
          }
      load_w(p);
    }
    if (last) {
      done(acc);
      clear(acc);
    }
    if (!more) break;
    store_b(buf + (turn ^ 1) * kSlab);
    wait_lgkm0();
    raw_barrier();
  }
}

// This thread's columns of an entry: `row(place)` is the byte offset of a place's
// activations; places past the entry's are kOutside.
template <int SG, int C, int H, typename Row>
__device__ __forceinline__ void aim_columns(uint32_t (&col)[H][C], int n, int p0, uint32_t plane, Row row) {
  constexpr int kCols = kRowWaves * kWave / (SG * 8);
  constexpr int kPer = C * 16 / kCols;   // of each plane
  static_assert(kPer <= C, "a thread's columns");
#pragma unroll
  for (int q = 0; q < H; ++q)
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int j = i * kCols + static_cast<int>(threadIdx.x) / (SG * 8);
      col[q][i] = i < kPer && j < n ? row(p0 + j) + q * plane : kOutside;
    }
}

// Units of one entry and 128 M gate and up rows, 16 M of each per wavefront, for
// the entries e0 .. e1 - 1 (all of C tiles).  Workgroup `me` of `grid` takes every
// grid-th unit, counted on from the `dealt` units before; returns the units dealt.
template <typename T, int C, int SG, int M, typename Places>
__device__ __forceinline__ int up_rows(const MoeArgs& a, const Places& pl, int e0, int e1, int dealt, int me, int grid,
                                       unsigned char* buf) {
  constexpr int kRows = 16 * M * kRowWaves;
  constexpr int R = 2 * M;
  const int lane = threadIdx.x % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t rb = static_cast<uint32_t>(a.d) * sizeof(T);
  const int blocks = (a.f + kRows - 1) / kRows;
  const int slabs = static_cast<int>((rb + SG * RowPairs::kBytes - 1) / (SG * RowPairs::kBytes));
  const int units = (e1 - e0) * blocks;
  const int u = (me - dealt % grid + grid) % grid;
  const size_t slot_bytes = static_cast<size_t>(3) * a.d * a.f * sizeof(T);
  int at = u;      // the unit of the slab set last,
  int i = -1;      // and that slab among the unit's
  int turn = 0;    // (rows of a power of two bytes: blocks start at different places)
  int unit = u;    // of the sums
  auto next = [&](Slab<C, 1, R>& s) __attribute__((always_inline)) {
    if (++i == slabs) {
      i = 0;
      at += grid;
    }
    if (at >= units) return false;
    if (i == 0) {   // (the unit's other slabs find this set)
      const int e = e0 + Places::entry(at, blocks, e1 - e0);
      const int blk = Places::block(at, blocks, e1 - e0);
      s.w = row_buffer(a.slots + __builtin_amdgcn_readfirstlane(pl.entry_slot[e]) * slot_bytes,
                       static_cast<uint32_t>(slot_bytes));
#pragma unroll
      for (int m = 0; m < M; ++m) {
        s.rows[m] = RowPairs(blk * kRows + 16 * (wv * M + m), a.f, rb, 0u);
        s.rows[M + m] = RowPairs(blk * kRows + 16 * (wv * M + m), a.f, rb, static_cast<uint32_t>(a.f) * rb);
      }
      aim_columns<SG>(s.col, pl.entry_n[e], pl.entry_place[e], 0u,
                      [&](int p) { return static_cast<uint32_t>(pl.token(p)) * rb; });
      turn = static_cast<int>(static_cast<uint32_t>(blk) * 5u % static_cast<uint32_t>(slabs));
    }
    const int q = i + turn < slabs ? i + turn : i + turn - slabs;
    s.k = static_cast<uint32_t>(q) * (SG * RowPairs::kBytes);
    s.k_end = rb;
    s.last = i + 1 == slabs;
    return true;
  };
  auto done = [&](floatx4 (&acc)[R][C]) __attribute__((always_inline)) {
    const int e = e0 + Places::entry(unit, blocks, e1 - e0);
    const int row0 = Places::block(unit, blocks, e1 - e0) * kRows + 16 * wv * M + 4 * (lane / 16);
    unit += grid;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int col = 16 * j + lane % 16;
      if (col >= pl.entry_n[e]) continue;
      const int place = pl.entry_place[e] + col;
      const float w = pl.weight_of(place);
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int row = row0 + 16 * m;
        if (row >= a.f) continue;   // (f is a multiple of 8: four rows exist or none does)
        floatx4 hv;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float gv = acc[m][j][r];
          hv[r] = w * (gv / (1.0f + expf(-gv)) * acc[M + m][j][r]);
        }
        store_h<T>(a, place, row, hv);
      }
    }
  };
  stream_slabs<T, C, 1, R, SG>(row_buffer(a.x, static_cast<uint32_t>(a.T) * rb), buf, next, done);
  return dealt + units;
}

constexpr int slab_bytes(int C, int H, int SG) { return 2 * H * C * 16 * (SG * 128 + 16); }

template <typename T>
__global__ void __launch_bounds__(kRowWaves * kWave, 4) k_moe_up_rows(MoeArgs a) {
  __shared__ Plan<kMoeTokens> pl;
  __shared__ __align__(16) unsigned char buf[slab_bytes(4, 1, 2) > slab_bytes(2, 1, 4) ? slab_bytes(4, 1, 2) : slab_bytes(2, 1, 4)];
  make_plan<kMoeTokens, kRowWaves * kWave>(a, pl);
  const int me = static_cast<int>(blockIdx.x), grid = static_cast<int>(gridDim.x);
  int dealt = up_rows<T, 1, 4, 1>(a, pl, 0, pl.classes[0], 0, me, grid, buf);
  dealt = up_rows<T, 2, 4, 1>(a, pl, pl.classes[0], pl.classes[1], dealt, me, grid, buf);
  up_rows<T, 4, 2, 1>(a, pl, pl.classes[1], pl.classes[2], dealt, me, grid, buf);
}

// Load groups [u, u1) of the concatenated entries, those among entries e0 .. e1 - 1
// (all of C tiles), for the workgroup's 128 R output rows, added to sums[t][128 R].
template <typename T, int C, int R, int SG>
__device__ __forceinline__ void down_rows(const MoeArgs& a, const Plan<kMoeTokens>& pl, int e0, int e1, int row0,
                                          int groups, int64_t share_u0, int64_t share_u1, float* sums,
                                          unsigned char* buf) {
  constexpr int H = sizeof(T) == 2 ? 2 : 1;   // planes of h
  constexpr int kRows = 16 * R * kRowWaves;
  const int lane = threadIdx.x % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t rb = static_cast<uint32_t>(a.f) * sizeof(T);
  const uint32_t plane = static_cast<uint32_t>(a.T) * a.K * rb;
  const int64_t lo = static_cast<int64_t>(e0) * groups, hi = static_cast<int64_t>(e1) * groups;
  int u = static_cast<int>(share_u0 > lo ? share_u0 : lo);
  const int u1 = static_cast<int>(share_u1 < hi ? share_u1 : hi);
  const size_t slot_elems = static_cast<size_t>(3) * a.d * a.f;
  const uint32_t down_bytes = static_cast<uint32_t>(static_cast<size_t>(a.d) * a.f * sizeof(T));
  RowPairs rows[R];
#pragma unroll
  for (int r = 0; r < R; ++r) rows[r] = RowPairs(row0 + 16 * (wv * R + r), a.d, rb, 0u);
  int at = u;          // first group of the next slab
  int entry = u / groups;   // of the sums
  auto next = [&](Slab<C, H, R>& s) __attribute__((always_inline)) {
    if (at >= u1) return false;
    const int e = at / groups;
    const int m0 = at - e * groups;
    const int end = (e + 1) * groups < u1 ? (e + 1) * groups : u1;   // of the entry's groups
    s.w = row_buffer(a.slots + (__builtin_amdgcn_readfirstlane(pl.entry_slot[e]) * slot_elems +
                                static_cast<size_t>(2) * a.d * a.f) * sizeof(T), down_bytes);
#pragma unroll
    for (int r = 0; r < R; ++r) s.rows[r] = rows[r];
    aim_columns<SG>(s.col, pl.entry_n[e], pl.entry_place[e], plane,
                    [&](int p) { return static_cast<uint32_t>(p) * rb; });
    s.k = static_cast<uint32_t>(m0) * RowPairs::kBytes;
    const uint32_t k_end = static_cast<uint32_t>(m0 + end - at) * RowPairs::kBytes;
    s.k_end = k_end < rb ? k_end : rb;
    at = at + SG < end ? at + SG : end;
    s.last = at == end;
    return true;
  };
  auto done = [&](floatx4 (&acc)[R][C]) __attribute__((always_inline)) {
    const int n = pl.entry_n[entry], p0 = pl.entry_place[entry];
    ++entry;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int col = 16 * j + lane % 16;
      if (col >= n) continue;
      float* o = sums + pl.tok[p0 + col] * kRows + 16 * R * wv + 4 * (lane / 16);
#pragma unroll
      for (int r = 0; r < R; ++r) *reinterpret_cast<floatx4*>(o + 16 * r) += acc[r][j];
    }
  };
  const uint32_t h_bytes = static_cast<uint32_t>(static_cast<size_t>(a.T) * a.K * a.f * 4);
  stream_slabs<T, C, H, R, SG>(row_buffer(a.h, h_bytes), buf, next, done);
}

// A workgroup owns 128 R output rows and one of the splits' shares of the load
// groups of all entries; its sums by token go to the split's partial sums.
template <typename T, int R>
__global__ void __launch_bounds__(kRowWaves * kWave, 2) k_moe_down_rows(MoeArgs a) {
  constexpr int H = sizeof(T) == 2 ? 2 : 1;
  constexpr int kRows = 16 * R * kRowWaves;
  constexpr int S2 = slab_bytes(2, H, 4), S4 = slab_bytes(4, H, 2);
  __shared__ Plan<kMoeTokens> pl;
  __shared__ __align__(16) unsigned char buf[S2 > S4 ? S2 : S4];
  extern __shared__ __align__(16) unsigned char smem[];   // [T][kRows] float32
  float* sums = reinterpret_cast<float*>(smem);
  const int tid = threadIdx.x;
  const int rbk = static_cast<int>(blockIdx.x) / a.splits;
  const int split = static_cast<int>(blockIdx.x) % a.splits;
  const int row0 = rbk * kRows;
  for (int i = tid; i < a.T * kRows / 4; i += kRowWaves * kWave)
    reinterpret_cast<floatx4*>(sums)[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  make_plan<kMoeTokens, kRowWaves * kWave>(a, pl);
  const int groups = (a.f * static_cast<int>(sizeof(T)) + kGroupBytes - 1) / kGroupBytes;
  const int64_t total = static_cast<int64_t>(pl.classes[2]) * groups;
  const int64_t u0 = total * split / a.splits;
  const int64_t u1 = total * (split + 1) / a.splits;
  down_rows<T, 1, R, 4>(a, pl, 0, pl.classes[0], row0, groups, u0, u1, sums, buf);
  down_rows<T, 2, R, 4>(a, pl, pl.classes[0], pl.classes[1], row0, groups, u0, u1, sums, buf);
  down_rows<T, 4, R, 2>(a, pl, pl.classes[1], pl.classes[2], row0, groups, u0, u1, sums, buf);
  __syncthreads();
  for (int i = tid; i < a.T * kRows / 4; i += kRowWaves * kWave) {
    const int t = i / (kRows / 4);
    const int row = row0 + 4 * (i % (kRows / 4));
    if (row < a.d)
      *reinterpret_cast<floatx4*>(a.partial + (static_cast<int64_t>(split) * a.T + t) * a.d + row) =
          reinterpret_cast<floatx4*>(sums)[i];
  }
}

// The splits' partial sums, in order, and the residual.
template <typename T>
__global__ void __launch_bounds__(256) k_moe_join(MoeArgs a) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  const int64_t n = static_cast<int64_t>(a.T) * a.d;
  if (i >= n) return;
  floatx4 v = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < a.splits; ++s) v += *reinterpret_cast<const floatx4*>(a.partial + s * n + i);
  store_out<T>(a, i, v);
}

// ---------------------------------------------------------------- long batches

// Above kMoeTokens an expert in use meets so many tokens that the matrix
// instructions, not the weights' stream, come to bound the products.  The same
// slabs then serve 64 weight rows per wavefront by 128 places: a piece of
// activations out of LDS feeds four matrix instructions, a weight eight.  The
// places are listed once, by a launch of one workgroup, and each place's product
// is written by itself; a last launch adds a token's K.
//
// 2,048 tokens, two each of 16 experts of 4,096 x 6,400, bf16: 1.10 ms, 584 TFLOP/s
// (779 with the products of h's second plane; the matrix units work 43-48% of the
// time); 4,096 tokens 1.87 ms.  A slab and CU load 160 KB, 2.1 us in pairs of lanes,
// and multiply for 1.7 us.  Few tokens' kernels against these: 64 tokens through 8
// of 4,096 x 14,336 478 and 589 us, 128 through 16 of 4,096 x 6,400 439 and 433, in
// float32 100 through 24 of 2,048 x 1,408 189 and 206.
constexpr int kLongPlaces = 128;   // of an entry
constexpr int kLongEntries = kMaxE + kLongTokens * kMaxK / kLongPlaces;

struct LongPlan {
  int32_t classes[4];   // ends of the entries of 1, 2, 4 and 8 tiles
  int32_t slot[kLongEntries], place[kLongEntries], n[kLongEntries];
};
struct LongArgs {
  MoeArgs m;
  LongPlan* plan;
  uint16_t* pair_of;    // [T K] pair (T, K) of each place
  int32_t* place_of;    // [T][K] (-1: no product)
};

constexpr int kListWaves = 16;
constexpr uint16_t kNone = 0xFFFF;   // (a wavefront's pairs: at most 2,048)

__global__ void __launch_bounds__(kListWaves * kWave) k_moe_list(LongArgs a) {
  __shared__ int32_t count[kListWaves][kMaxE];   // then the next place of each wavefront's share
  __shared__ int32_t slot[kMaxE];
  // each pair's rank among its wavefront's of the expert, then each place's pair
  extern __shared__ __align__(16) uint16_t rank[];   // [2][T K], each rounded up to 16 bytes
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = tid / kWave;
  const int pairs = a.m.T * a.m.K;
  uint16_t* pair_of = rank + (pairs + 7) / 8 * 8;
  if (tid < kMaxE) slot[tid] = tid < a.m.E ? a.m.slot_of[tid] : -1;
  count[wv][lane] = 0;
  __syncthreads();
  const int share = (pairs + kListWaves * kWave - 1) / (kListWaves * kWave) * kWave;
  const int p0 = wv * share;
  const int p1 = p0 + share < pairs ? p0 + share : pairs;
  constexpr int U = 4;   // steps of 64 pairs whose loads go out together
  uint32_t bad = 0;
  for (int q = p0; q < p1; q += U * kWave) {
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = q + u * kWave + lane < p1 ? a.m.ids[q + u * kWave + lane] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = q + u * kWave + lane;
      if (q + u * kWave >= p1) break;
      int e = id[u];
      if (e >= 0) {
        const int s = e < a.m.E ? slot[e] : 0;
        const uint32_t b = e >= a.m.E || s >= a.m.n_slots ? FM_FLAG_INDEX_RANGE : (s < 0 ? FM_FLAG_EXPERT_MISSING : 0);
        bad |= b;
        if (b != 0) e = -1;
      }
      // the lanes that hold the same expert; the first of them counts for all
      uint64_t m = __ballot(e >= 0);
#pragma unroll
      for (int b = 0; b < 6; ++b) {
        const bool bit = (e >> b & 1) != 0;
        const uint64_t one = __ballot(bit);
        m &= bit ? one : ~one;
      }
      if (p >= p1) continue;
      const int before = __popcll(m & ((1ull << lane) - 1ull));
      if (e < 0) {
        rank[p] = kNone;
        continue;
      }
      // (a wavefront's LDS accesses happen in its order: every lane reads before
      // the first one adds)
      volatile int32_t* c = &count[wv][e];
      const int n = *c;
      rank[p] = static_cast<uint16_t>(n + before);
      if (before == 0) *c = n + __popcll(m);
    }
  }
  if (bad != 0 && a.m.flags != nullptr) atomicOr(a.m.flags, bad);
  __syncthreads();
  if (wv == 0) {   // an expert per lane
    int n = 0;
    for (int w = 0; w < kListWaves; ++w) n += count[w][lane];
    auto scan = [&](int v) {   // exclusive
      int incl = v;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int u = __shfl_up(incl, o, kWave);
        if (lane >= o) incl += u;
      }
      return incl - v;
    };
    const int first = scan(n);
    int next = first;
    for (int w = 0; w < kListWaves; ++w) {
      const int c = count[w][lane];
      count[w][lane] = next;
      next += c;
    }
    const int rest = n % kLongPlaces;
    int base = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      // entries of this class: of the last one the expert's rest, and the whole ones
      const bool mine = rest > (c == 0 ? 0 : 8 << c) && rest <= (c == 3 ? kLongPlaces : 16 << c);
      const int have = (mine ? 1 : 0) + (c == 3 ? n / kLongPlaces : 0);
      const int at = base + scan(have);
      for (int j = 0; j < have; ++j) {
        const int from = mine && j + 1 == have ? n - rest : j * kLongPlaces;
        a.plan->slot[at + j] = slot[lane];
        a.plan->place[at + j] = first + from;
        a.plan->n[at + j] = n - from < kLongPlaces ? n - from : kLongPlaces;
      }
      base = __shfl(at + have, kWave - 1, kWave);
      if (lane == 0) a.plan->classes[c] = base;
    }
  }
  __syncthreads();
#pragma unroll 4
  for (int p = p0 + lane; p < p1; p += kWave) {
    const int e = a.m.ids[p];
    const int at = rank[p] != kNone ? count[wv][e] + rank[p] : -1;
    a.place_of[p] = at;
    if (at >= 0) pair_of[at] = static_cast<uint16_t>(p);
  }
  __syncthreads();
  // (written here in order: places in the pairs' order scatter, and one CU's stores
  // take a clock per lane then)
  for (int i = tid; i < (pairs + 1) / 2; i += kListWaves * kWave)
    reinterpret_cast<uint32_t*>(a.pair_of)[i] = reinterpret_cast<const uint32_t*>(pair_of)[i];
}

// The list as the products' kernels see it: the entries (and for the gate and up
// projections the pairs) in LDS, read in every unit.
struct LongPlaces {
  const int32_t *entry_slot, *entry_place, *entry_n;
  const uint16_t* pair_of;
  const float* weights;   // [T][K]
  int K;
  __device__ __forceinline__ int token(int place) const { return pair_of[place] / K; }
  __device__ __forceinline__ float weight_of(int place) const { return weights[pair_of[place]]; }
  // the entries vary fastest: an expert's are neighbours and read the same
  // weights, in workgroups of one XCD at the same time
  static __device__ __forceinline__ int entry(int u, int, int n) { return u % n; }
  static __device__ __forceinline__ int block(int u, int, int n) { return u / n; }
};

constexpr int kXcds = 8;
// Consecutive workgroups go to different XCDs; this numbers those of an XCD in a
// row, so that an expert's entries share its L2 (2,048 tokens through 8 experts of
// 4,096 x 14,336: 2.43 -> 2.04 ms).
__device__ __forceinline__ int xcd_order() {
  return static_cast<int>(blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds);
}

template <int H>
constexpr int long_slab() {
  constexpr int a = slab_bytes(4, H, 4), b = slab_bytes(8, H, 2);
  return a > b ? a : b;
}

// Whether units of twice `rows` rows end sooner: per row they cost three quarters
// (an activation out of LDS feeds four matrix instructions instead of two), but
// there are half as many to deal among the workgroups.
__device__ __forceinline__ bool wide_units(int entries, int all_rows, int rows, int grid) {
  auto turns = [&](int n) { return (entries * ((all_rows + n - 1) / n) + grid - 1) / grid; };
  return 3 * turns(2 * rows) <= 2 * turns(rows);
}

// The entries from the plan into LDS.
__device__ __forceinline__ void stage_entries(const LongPlan& plan, int32_t (*e)[kLongEntries]) {
  const int n = plan.classes[3];
  for (int i = threadIdx.x; i < n; i += kRowWaves * kWave) {
    e[0][i] = plan.slot[i];
    e[1][i] = plan.place[i];
    e[2][i] = plan.n[i];
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowWaves * kWave, 2) k_moe_up_long(LongArgs a) {
  __shared__ int32_t entries[3][kLongEntries];
  extern __shared__ __align__(16) unsigned char smem[];   // [slabs][pairs of the places]
  uint32_t* pairs = reinterpret_cast<uint32_t*>(smem + long_slab<1>());
  stage_entries(*a.plan, entries);
  for (int i = threadIdx.x; i < (a.m.T * a.m.K + 1) / 2; i += kRowWaves * kWave)
    pairs[i] = reinterpret_cast<const uint32_t*>(a.pair_of)[i];
  __syncthreads();
  const LongPlaces pl{entries[0], entries[1], entries[2], reinterpret_cast<const uint16_t*>(pairs), a.m.weight, a.m.K};
  const int32_t* cl = a.plan->classes;
  const int me = xcd_order(), grid = static_cast<int>(gridDim.x);
  int dealt;
  if (wide_units(cl[3] - cl[2], a.m.f, 16 * kRowWaves, grid))
    dealt = up_rows<T, 8, 2, 2>(a.m, pl, cl[2], cl[3], 0, me, grid, smem);
  else
    dealt = up_rows<T, 8, 2, 1>(a.m, pl, cl[2], cl[3], 0, me, grid, smem);
  dealt = up_rows<T, 4, 4, 1>(a.m, pl, cl[1], cl[2], dealt, me, grid, smem);
  dealt = up_rows<T, 2, 4, 1>(a.m, pl, cl[0], cl[1], dealt, me, grid, smem);
  up_rows<T, 1, 4, 1>(a.m, pl, 0, cl[0], dealt, me, grid, smem);
}

// Units of one entry and 128 R output rows, 16 R per wavefront, dealt as up_rows
// deals them; each place's product goes to its own row.
template <typename T, int C, int R, int SG>
__device__ __forceinline__ int down_long(const MoeArgs& a, const LongPlaces& pl, int e0, int e1, int dealt, int me,
                                         int grid, unsigned char* buf) {
  constexpr int H = sizeof(T) == 2 ? 2 : 1;   // planes of h
  constexpr int kRows = 16 * R * kRowWaves;
  const int lane = threadIdx.x % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t rb = static_cast<uint32_t>(a.f) * sizeof(T);
  const uint32_t plane = static_cast<uint32_t>(a.T) * a.K * rb;
  const int blocks = (a.d + kRows - 1) / kRows;
  const int slabs = static_cast<int>((rb + SG * RowPairs::kBytes - 1) / (SG * RowPairs::kBytes));
  const int units = (e1 - e0) * blocks;
  const int u = (me - dealt % grid + grid) % grid;
  const size_t slot_elems = static_cast<size_t>(3) * a.d * a.f;
  const uint32_t down_bytes = static_cast<uint32_t>(static_cast<size_t>(a.d) * a.f * sizeof(T));
  int at = u, i = -1, turn = 0, unit = u;
  auto next = [&](Slab<C, H, R>& s) __attribute__((always_inline)) {
    if (++i == slabs) {
      i = 0;
      at += grid;
    }
    if (at >= units) return false;
    if (i == 0) {
      const int e = e0 + LongPlaces::entry(at, blocks, e1 - e0);
      const int blk = LongPlaces::block(at, blocks, e1 - e0);
      s.w = row_buffer(a.slots + (__builtin_amdgcn_readfirstlane(pl.entry_slot[e]) * slot_elems +
                                  static_cast<size_t>(2) * a.d * a.f) * sizeof(T), down_bytes);
#pragma unroll
      for (int r = 0; r < R; ++r) s.rows[r] = RowPairs(blk * kRows + 16 * (wv * R + r), a.d, rb, 0u);
      aim_columns<SG>(s.col, pl.entry_n[e], pl.entry_place[e], plane,
                      [&](int p) { return static_cast<uint32_t>(p) * rb; });
      turn = static_cast<int>(static_cast<uint32_t>(blk) * 5u % static_cast<uint32_t>(slabs));
    }
    const int q = i + turn < slabs ? i + turn : i + turn - slabs;
    s.k = static_cast<uint32_t>(q) * (SG * RowPairs::kBytes);
    s.k_end = rb;
    s.last = i + 1 == slabs;
    return true;
  };
  auto done = [&](floatx4 (&acc)[R][C]) __attribute__((always_inline)) {
    const int e = e0 + LongPlaces::entry(unit, blocks, e1 - e0);
    const int row0 = LongPlaces::block(unit, blocks, e1 - e0) * kRows + 16 * R * wv + 4 * (lane / 16);
    unit += grid;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int col = 16 * j + lane % 16;
      if (col >= pl.entry_n[e]) continue;
      float* o = a.partial + static_cast<int64_t>(pl.entry_place[e] + col) * a.d + row0;
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (row0 + 16 * r < a.d) *reinterpret_cast<floatx4*>(o + 16 * r) = acc[r][j];
    }
  };
  const uint32_t h_bytes = static_cast<uint32_t>(static_cast<size_t>(a.T) * a.K * a.f * 4);
  stream_slabs<T, C, H, R, SG>(row_buffer(a.h, h_bytes), buf, next, done);
  return dealt + units;
}

template <typename T>
__global__ void __launch_bounds__(kRowWaves * kWave, 2) k_moe_down_long(LongArgs a) {
  __shared__ int32_t entries[3][kLongEntries];
  extern __shared__ __align__(16) unsigned char smem[];   // slabs
  stage_entries(*a.plan, entries);
  __syncthreads();
  const LongPlaces pl{entries[0], entries[1], entries[2], nullptr, nullptr, 0};
  const int32_t* cl = a.plan->classes;
  const int me = xcd_order(), grid = static_cast<int>(gridDim.x);
  int dealt;
  if (wide_units(cl[3] - cl[2], a.m.d, 32 * kRowWaves, grid))
    dealt = down_long<T, 8, 4, 2>(a.m, pl, cl[2], cl[3], 0, me, grid, smem);
  else
    dealt = down_long<T, 8, 2, 2>(a.m, pl, cl[2], cl[3], 0, me, grid, smem);
  dealt = down_long<T, 4, 2, 4>(a.m, pl, cl[1], cl[2], dealt, me, grid, smem);
  dealt = down_long<T, 2, 2, 4>(a.m, pl, cl[0], cl[1], dealt, me, grid, smem);
  down_long<T, 1, 2, 4>(a.m, pl, 0, cl[0], dealt, me, grid, smem);
}

// A token's products, in the order of its experts, and the residual.
template <typename T>
__global__ void __launch_bounds__(256) k_moe_sum(LongArgs a) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= static_cast<int64_t>(a.m.T) * a.m.d) return;
  const int t = static_cast<int>(i / a.m.d);
  const int row = static_cast<int>(i - static_cast<int64_t>(t) * a.m.d);
  floatx4 v = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < a.m.K; ++k) {
    const int p = a.place_of[t * a.m.K + k];
    if (p >= 0) v += *reinterpret_cast<const floatx4*>(a.m.partial + static_cast<int64_t>(p) * a.m.d + row);
  }
  store_out<T>(a.m, i, v);
}

// ---------------------------------------------------------------- host

constexpr int kCus = 256;
constexpr int kFewTokens = 16;   // up to here the wavefronts of a workgroup split the long axis

// How k_moe_down (few tokens) or k_moe_down_rows cuts the output.
struct DownShape {
  int rows;     // per workgroup
  int blocks;   // of rows
  int splits;   // shares of the experts' products, so that the workgroups fill the GPU
};
DownShape down_shape(int32_t d, int32_t T) {
  DownShape s;
  s.rows = T <= kFewTokens ? 32 : (T <= 64 ? 256 : 128);   // (sums by token of up to 64 KB)
  s.blocks = (d + s.rows - 1) / s.rows;
  const int want = T <= kFewTokens ? 2 * kCus : kCus;
  s.splits = (want + s.blocks - 1) / s.blocks;
  const int most = T <= kFewTokens ? 16 : 64;
  if (s.splits > most) s.splits = most;
  return s;
}

template <typename T>
hipError_t few_tokens(const MoeArgs& a, hipStream_t st) {
  // at most this many units; each workgroup takes its turn at them
  const int experts = a.E < a.T * a.K ? a.E : a.T * a.K;
  const int units = experts * ((a.f + kUpRows - 1) / kUpRows);
  k_moe_up<T><<<static_cast<unsigned>(units < 2 * kCus ? units : 2 * kCus), kUpWaves * kWave, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_moe_down<T><<<static_cast<unsigned>(a.row_blocks) * static_cast<unsigned>(a.splits), kDownWaves * kWave, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T, int R>
hipError_t more_tokens(const MoeArgs& a, hipStream_t st) {
  const int experts = a.E + a.T * a.K / 64 < a.T * a.K ? a.E + a.T * a.K / 64 : a.T * a.K;   // entries, at most
  const int units = experts * ((a.f + 16 * kRowWaves - 1) / (16 * kRowWaves));
  k_moe_up_rows<T><<<static_cast<unsigned>(units < 2 * kCus ? units : 2 * kCus), kRowWaves * kWave, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto kern = k_moe_down_rows<T, R>;
  const size_t lds = static_cast<size_t>(a.T) * 16 * R * kRowWaves * sizeof(float);
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(lds));
  if (e != hipSuccess) return e;
  kern<<<static_cast<unsigned>(a.row_blocks) * static_cast<unsigned>(a.splits), kRowWaves * kWave, lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t quads = static_cast<int64_t>(a.T) * a.d / 4;
  k_moe_join<T><<<static_cast<unsigned>((quads + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t long_batch(const LongArgs& a, hipStream_t st) {
  constexpr int H = sizeof(T) == 2 ? 2 : 1;
  const size_t up_lds = long_slab<1>() + align_up(static_cast<size_t>(a.m.T) * a.m.K * sizeof(uint16_t), 16);
  const size_t down_lds = long_slab<H>();
  auto up = k_moe_up_long<T>;
  auto down = k_moe_down_long<T>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(up), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(up_lds));
  if (e != hipSuccess) return e;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(down), hipFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(down_lds));
  if (e != hipSuccess) return e;
  const size_t list_lds = align_up(static_cast<size_t>(a.m.T) * a.m.K * sizeof(uint16_t), 16) * 2;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_moe_list), hipFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(list_lds));
  if (e != hipSuccess) return e;
  k_moe_list<<<1, kListWaves * kWave, list_lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  up<<<kCus, kRowWaves * kWave, up_lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  down<<<kCus, kRowWaves * kWave, down_lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t quads = static_cast<int64_t>(a.m.T) * a.m.d / 4;
  k_moe_sum<T><<<static_cast<unsigned>((quads + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t experts(const MoeArgs& a, hipStream_t st) {
  if (a.T <= kFewTokens) return few_tokens<T>(a, st);
  return a.T <= 64 ? more_tokens<T, 2>(a, st) : more_tokens<T, 1>(a, st);
}

// Tokens of one pass of a long batch: as many as 256 MB hold of h and of the
// places' products (the weights in use are read once per pass).
int32_t long_tokens(int32_t d, int32_t f, int32_t K) {
  const int64_t fit = (int64_t{1} << 28) / (static_cast<int64_t>(K) * (d > f ? d : f) * 4);
  return fit < kLongTokens ? static_cast<int32_t>(fit) : kLongTokens;
}

// Workspace of one launch, its parts 256-byte aligned: [h][tickets][partial sums],
// or of a long batch [h][plan][places' pairs][pairs' places][products].
struct Parts {
  size_t ticket, partial, plan, pair_of, place_of, bytes;
};
Parts parts(int32_t d, int32_t f, int32_t T, int32_t K) {
  Parts p = {};
  const size_t pairs = static_cast<size_t>(T) * K;
  size_t at = align_up(pairs * f * 4, kAlign);
  auto take = [&](size_t n) {
    const size_t o = at;
    at += align_up(n, kAlign);
    return o;
  };
  if (T <= kMoeTokens) {
    p.ticket = take(static_cast<size_t>((d + 31) / 32) * sizeof(uint32_t));
    p.partial = take(static_cast<size_t>(down_shape(d, T).splits) * T * d * sizeof(float));
  } else {
    p.plan = take(sizeof(LongPlan));
    p.pair_of = take((pairs + 1) / 2 * sizeof(uint32_t));
    p.place_of = take(pairs * sizeof(int32_t));
    p.partial = take(pairs * d * sizeof(float));
  }
  p.bytes = at;
  return p;
}

}  // namespace

size_t moe_workspace_bytes(int32_t d, int32_t f, fm_dtype, int32_t T, int32_t K) {
  // what the largest launch needs, and any smaller one; a long batch always gets
  // a whole launch's, so that one size serves all of them
  size_t most = T > kMoeTokens ? parts(d, f, long_tokens(d, f, K), K).bytes : 0;
  for (int32_t t : {kFewTokens, 64, kMoeTokens}) {
    const size_t n = parts(d, f, T < t ? T : t, K).bytes;
    most = n > most ? n : most;
  }
  return most;
}

hipError_t launch_moe_experts(const fm_expert_cache& c, const void* x, const int32_t* ids, const float* weight,
                              int32_t T, int32_t K, const void* residual, void* out, uint32_t* flags, void* ws,
                              hipStream_t st) {
  const size_t es = c.dtype == FM_BF16 ? 2 : 4;
  const size_t row = static_cast<size_t>(c.d) * es;
  const int32_t most = long_tokens(c.d, c.f, K);
  char* base = static_cast<char*>(ws);
  for (int32_t t0 = 0; t0 < T; t0 += most) {
    LongArgs l;
    MoeArgs& a = l.m;
    a.T = T - t0 < most ? T - t0 : most;
    const Parts p = parts(c.d, c.f, a.T, K);
    const DownShape s = down_shape(c.d, a.T);
    a.slots = static_cast<const char*>(c.slots);
    a.slot_of = c.slot_of;
    a.x = static_cast<const char*>(x) + t0 * row;
    a.ids = ids + static_cast<int64_t>(t0) * K;
    a.weight = weight + static_cast<int64_t>(t0) * K;
    a.residual = residual == nullptr ? nullptr : static_cast<const char*>(residual) + t0 * row;
    a.out = static_cast<char*>(out) + t0 * row;
    a.h = base;
    a.partial = reinterpret_cast<float*>(base + p.partial);
    a.ticket = reinterpret_cast<uint32_t*>(base + p.ticket);
    a.flags = flags;
    a.K = K;
    a.E = c.E;
    a.n_slots = c.n_slots;
    a.d = c.d;
    a.f = c.f;
    a.splits = s.splits;
    a.row_blocks = s.blocks;
    hipError_t e;
    if (a.T <= kMoeTokens) {
      e = c.dtype == FM_BF16 ? experts<uint16_t>(a, st) : experts<float>(a, st);
    } else {
      l.plan = reinterpret_cast<LongPlan*>(base + p.plan);
      l.pair_of = reinterpret_cast<uint16_t*>(base + p.pair_of);
      l.place_of = reinterpret_cast<int32_t*>(base + p.place_of);
      e = c.dtype == FM_BF16 ? long_batch<uint16_t>(l, st) : long_batch<float>(l, st);
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fm
