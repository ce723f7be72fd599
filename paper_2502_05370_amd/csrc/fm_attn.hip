// Attention of one new token per slot over the pages of its sequence.
//
// A wavefront takes 32 tokens (float32: 16) of a key head at a time, for up to 16
// query heads that read it.  The pages hold operands: a piece of 1 KB is one load
// of 16 bytes a lane, whole lines, and the very registers that the matrix
// instructions take.
//   scores   S^T = K Q^T: rows are tokens, columns are queries.  Lane 16 g + c gets
//            tokens 4 g .. 4 g + 3 of each block of 16, for query c.
//   output   O^T += V^T P^T: the same lane must hold P of query c for four tokens
//            per block, which are the ones it has, so that the probabilities pass
//            from accumulators to operands without changing lanes.
// Running maximum and sum per query; the sums and outputs are scaled only when a
// maximum has grown.  Memory bounds it: 16 queries per key head cost the matrix
// units 7% of the time that the keys and values take to arrive.
#include "fm_device.h"
#include "fm_kv.h"
#include "fm_mma.h"

namespace fm {

namespace {

constexpr int kAttnWaves = 4;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// Over the four lanes that share lane % 16.
__device__ __forceinline__ float max_of_groups(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_groups(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
}

// What p cut to `cut` leaves (NaN stays NaN in the cut part).
__device__ __forceinline__ float rest(float p, uint32_t cut) { return fmaxf(p - __uint_as_float(cut), 0x1p-126f); }

// The tokens that a slot's query sees.
struct Seen {
  int32_t lo, hi;   // places
  __device__ __forceinline__ bool none() const { return lo >= hi; }
};
__device__ __forceinline__ Seen seen_of(const AttnArgs& a, int s) {
  const int32_t len = a.c.tokens(a.c.length[s]);
  int32_t lo = a.first != nullptr ? a.first[s] : 0;
  lo = lo < 0 ? 0 : lo;
  if (a.window > 0 && len - a.window > lo) lo = len - a.window;
  if (a.active != nullptr && a.active[s] == 0) lo = len;
  return Seen{lo, len};
}

template <typename T, int NP>
struct Wave {
  static constexpr bool kBf = sizeof(T) == 2;
  static constexpr int SB = kBf ? 2 : 1;       // blocks of a step
  static constexpr int OT = NP * (kBf ? 2 : 1);   // tiles of 16 dimensions
  uint32x4 q[NP];
  uint32x4 k[SB][NP], v[SB][NP];
  floatx4 o[OT];
  float m, l;   // of query c; l: this lane's tokens

  __device__ __forceinline__ void clear() {
    m = -__builtin_inff();
    l = 0.0f;
#pragma unroll
    for (int t = 0; t < OT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  static __device__ __forceinline__ void load(const char* at, uint32x4 (&r)[NP]) {
    const uint32x4* p = reinterpret_cast<const uint32x4*>(at) + threadIdx.x % kWave;
#pragma unroll
    for (int t = 0; t < NP; ++t) r[t] = __builtin_nontemporal_load(p + t * (kPieceBytes / 16));
  }
  __device__ __forceinline__ void scores(floatx4 (&s)[SB]) const {
#pragma unroll
    for (int b = 0; b < SB; ++b) {
      s[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NP; ++t) s[b] = mma_step<T>(k[b][t], q[t], s[b]);
    }
  }
  // Scores to probabilities, in place.  MASK: tokens of block b outside [lo[b],
  // hi[b]) have no part, nor have their values.
  template <bool MASK>
  __device__ __forceinline__ void weigh(floatx4 (&s)[SB], float scale2, const int (&lo)[SB], const int (&hi)[SB]) {
    const int row = threadIdx.x % kWave / 16 * 4;
    float top = -__builtin_inff();
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float t = s[b][r] * scale2;
        if (MASK && !(row + r >= lo[b] && row + r < hi[b])) t = -__builtin_inff();
        top = fmaxf(top, t);
      }
    top = max_of_groups(top);
    if (__any(top > m)) {
      const float grown = fmaxf(m, top);
      // (a first maximum scales zeros; minus infinity stands for no score yet)
      const float f = grown > m ? __builtin_amdgcn_exp2f(m - grown) : 1.0f;
      m = grown;
      l *= f;
#pragma unroll
      for (int t = 0; t < OT; ++t) o[t] *= f;
    }
    const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], scale2, -base));
        if (MASK && !(row + r >= lo[b] && row + r < hi[b])) p = 0.0f;
        s[b][r] = p;
        l += p;
      }
    if constexpr (MASK) {
#pragma unroll
      for (int b = 0; b < SB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool in = row + r >= lo[b] && row + r < hi[b];
#pragma unroll
          for (int t = 0; t < NP; ++t) {
            if constexpr (kBf) {
              const uint32_t keep = in ? 0xFFFFFFFFu : (r % 2 == 0 ? 0xFFFF0000u : 0x0000FFFFu);
              v[b][t][r / 2] &= keep;
              v[b][t][2 + r / 2] &= keep;
            } else {
              v[b][t][r] = in ? v[b][t][r] : 0u;
            }
          }
        }
    }
  }
  __device__ __forceinline__ void add(const floatx4 (&p)[SB]) {
    if constexpr (kBf) {
      // p as two bf16, so that the result is off by its own rounding alone: p cut
      // towards zero, and the rest.  2^-126 stands for a rest of zero, so that an
      // infinite value gives infinity and not the NaN of infinity times zero.
      uint32x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = p[i / 2][i % 2 * 2], y = p[i / 2][i % 2 * 2 + 1];
        hi[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
        lo[i] = pack_bf16(rest(x, hi[i] << 16), rest(y, hi[i] & 0xFFFF0000u));
      }
#pragma unroll
      for (int t = 0; t < NP; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32x4 w = {v[0][t][2 * i], v[0][t][2 * i + 1], v[1][t][2 * i], v[1][t][2 * i + 1]};
          o[2 * t + i] = mma_step<T>(w, hi, o[2 * t + i]);
          o[2 * t + i] = mma_step<T>(w, lo, o[2 * t + i]);
        }
    } else {
#pragma unroll
      for (int t = 0; t < NP; ++t) o[t] = mma_step<T>(v[0][t], __builtin_bit_cast(uint32x4, p[0]), o[t]);
    }
  }
};

// A wavefront's steps [first, last) with a stride of a slot's blocks, counted from
// the block of the first visible token.
template <typename T, int NP>
__device__ __forceinline__ void walk(const AttnArgs& a, Wave<T, NP>& w, int slot, int head, Seen seen, int first,
                                     int last, int stride, uint32_t& bad) {
  using W = Wave<T, NP>;
  constexpr int SB = W::SB;
  const int per_page = a.c.page / kBlockTokens;
  const int block_bytes = NP * kPieceBytes;
  const int32_t* row = a.c.table + static_cast<int64_t>(slot) * a.c.max_pages;
  const char* keys = a.c.pages + a.c.head_offset(a.layer, 0, head);
  const int64_t to_values = a.c.head_offset(0, 1, 0);
  const int b0 = seen.lo / kBlockTokens;
  const int b1 = (seen.hi + kBlockTokens - 1) / kBlockTokens;

  // where block b lies, and which of its tokens are seen: none of one that does
  // not exist or whose page does not, which stands at another's place
  int base = 0, ids = 0;   // a page number per lane, of the table's entries from base on
  bool filled = false;
  auto locate = [&](int step, const char* (&at)[SB], int (&lo)[SB], int (&hi)[SB]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < SB; ++i) {
      const int b = b0 + step * SB + i;
      const int bb = b < b1 ? b : b1 - 1;
      const int entry = static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(bb)) * a.per_page_inv) >> 32);
      if (!filled || entry >= base + kWave) {
        base = entry;
        filled = true;
        const int mine = entry + static_cast<int>(threadIdx.x % kWave);
        ids = row[mine < a.c.max_pages ? mine : a.c.max_pages - 1];
      }
      int page = __builtin_amdgcn_readlane(ids, entry - base);
      lo[i] = seen.lo - b * kBlockTokens;
      hi[i] = b < b1 ? seen.hi - b * kBlockTokens : 0;
      if (!a.c.valid(page)) {
        bad = FM_FLAG_INDEX_RANGE;
        page = 0;
        hi[i] = 0;
      }
      at[i] = keys + page * a.c.page_bytes + static_cast<int64_t>(bb - entry * per_page) * block_bytes;
    }
  };
  const char* at[SB];
  int lo[SB], hi[SB];
  if (first >= last) return;
  locate(first, at, lo, hi);
#pragma unroll
  for (int i = 0; i < SB; ++i) W::load(at[i], w.k[i]);
#pragma unroll
  for (int i = 0; i < SB; ++i) W::load(at[i] + to_values, w.v[i]);
  for (int step = first; step < last; step += stride) {
    int lo0[SB], hi0[SB];   // of this step
#pragma unroll
    for (int i = 0; i < SB; ++i) {
      lo0[i] = lo[i];
      hi0[i] = hi[i];
    }
    const bool more = step + stride < last;
    floatx4 s[SB];
    w.scores(s);
    if (more) {
      locate(step + stride, at, lo, hi);
#pragma unroll
      for (int i = 0; i < SB; ++i) W::load(at[i], w.k[i]);
    }
    bool whole = true;
#pragma unroll
    for (int i = 0; i < SB; ++i) whole = whole && lo0[i] <= 0 && hi0[i] >= kBlockTokens;
    if (whole) w.template weigh<false>(s, a.scale2, lo0, hi0);
    else w.template weigh<true>(s, a.scale2, lo0, hi0);
    w.add(s);
    if (more) {
#pragma unroll
      for (int i = 0; i < SB; ++i) W::load(at[i] + to_values, w.v[i]);
    }
  }
}

// Queries of one key head and tile: lane 16 g + c holds 16 bytes of query c per 64.
template <typename T, int NP>
__device__ __forceinline__ void load_queries(const AttnArgs& a, Wave<T, NP>& w, int slot, int head, int tile) {
  constexpr int N = 16 / static_cast<int>(sizeof(T));
  const int lane = threadIdx.x % kWave;
  const int c = lane % 16 + tile * 16, g = lane / 16;
  const char* row = a.q + slot * a.q_row + static_cast<int64_t>(head * a.group + c) * a.c.head_dim * sizeof(T);
#pragma unroll
  for (int t = 0; t < NP; ++t) {
    const int d = 4 * N * t + N * g;
    w.q[t] = uint32x4{0u, 0u, 0u, 0u};
    if (c < a.group && d < a.c.head_dim)
      w.q[t] = *reinterpret_cast<const uint32x4*>(row + static_cast<int64_t>(d) * sizeof(T));
  }
}

template <typename T>
__device__ __forceinline__ void store4(char* out, int64_t i, floatx4 v) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint32x2*>(reinterpret_cast<T*>(out) + i) = uint32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  } else {
    *reinterpret_cast<floatx4*>(reinterpret_cast<T*>(out) + i) = v;
  }
}

// Maxima, sums and outputs of a tile's parts, through LDS.
template <int NP4>   // dimensions of a padded row
struct Joined {
  static constexpr int kLd = NP4 + 4;
  float m[kAttnWaves][16], l[kAttnWaves][16];
  float o[kAttnWaves][16][kLd];
};

// A part in the workspace: m [16], l [16], outputs [queries of a tile][padded row].
__host__ __device__ inline int64_t part_floats(int32_t group, int dims) {
  return 32 + static_cast<int64_t>(group < 16 ? group : 16) * dims;
}

__device__ __forceinline__ void put(float* p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float get(const float* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// How much of a part counts in a sum relative to the maximum `top`.  A part that saw
// no score has the maximum minus infinity, and one that saw only NaN too.
__device__ __forceinline__ float share(float m, float l, float top) {
  return m == -__builtin_inff() ? (l == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(m - top);
}

// The four entries of `sh` together: to the output, or as a part to the workspace.
template <typename T, int DIMS>
__device__ __forceinline__ void finish(const AttnArgs& a, const Joined<DIMS>& sh, int slot, int q0, int queries,
                                       float* part) {
  const int quads = a.c.head_dim / 4;
  for (int i = threadIdx.x; i < queries * quads; i += kAttnWaves * kWave) {
    const int qi = i / quads, d = i % quads * 4;
    float top = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) top = fmaxf(top, sh.m[u][qi]);
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    float all = 0.0f;
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) {
      const float f = share(sh.m[u][qi], sh.l[u][qi], top);
      all += f * sh.l[u][qi];
      sum += f * *reinterpret_cast<const floatx4*>(&sh.o[u][qi][d]);
    }
    if (part != nullptr) {
      if (d == 0) {
        put(part + qi, top);
        put(part + 16 + qi, all);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) put(part + 32 + qi * DIMS + d + r, sum[r]);
      continue;
    }
    const int64_t at = static_cast<int64_t>(slot) * a.q_heads + q0 + qi;
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    store4<T>(a.out, at * a.c.head_dim + d, all == 0.0f ? zero : sum / all);
    if (d == 0 && a.lse != nullptr)
      a.lse[at] = all == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(all)) * kLn2;
  }
}

// Parts first .. first + n - 1 of a tile (part(i) their addresses) into `sh`, a
// wavefront every fourth of them.
template <int DIMS, typename Part>
__device__ __forceinline__ void collect(const AttnArgs& a, Joined<DIMS>& sh, int queries, int n, Part part) {
  constexpr int U = 8;   // parts whose loads are in flight together
  const int lane = threadIdx.x % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int quads = a.c.head_dim / 4;
  for (int i = lane; i < queries * quads; i += kWave) {
    const int qi = i / quads, d = i % quads * 4;
    float m = -__builtin_inff(), l = 0.0f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = wv; p0 < n; p0 += U * kAttnWaves) {
      float pm[U], pl[U];
      floatx4 po[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = p0 + u * kAttnWaves;
        const float* at = part(p < n ? p : wv);
        pm[u] = get(at + qi);
        pl[u] = get(at + 16 + qi);
#pragma unroll
        for (int r = 0; r < 4; ++r) po[u][r] = get(at + 32 + qi * DIMS + d + r);
      }
      float top = m;
#pragma unroll
      for (int u = 0; u < U; ++u) top = p0 + u * kAttnWaves < n ? fmaxf(top, pm[u]) : top;
      const float f = share(m, l, top);
      l *= f;
      o *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p0 + u * kAttnWaves >= n) continue;
        const float g = share(pm[u], pl[u], top);
        l += g * pl[u];
        o += g * po[u];
      }
      m = top;
    }
    *reinterpret_cast<floatx4*>(&sh.o[wv][qi][d]) = o;
    if (d == 0) {
      sh.m[wv][qi] = m;
      sh.l[wv][qi] = l;
    }
  }
}

// The batch's work is a line: slot after slot, in it key head after key head (and
// tile after tile of its queries), in it kOverhead units and one per step.  Every
// workgroup takes as much of the line, whatever the lengths are.  What it has of a
// tile is a part; a tile of several workgroups is joined by the last of them that
// is done (tickets, no wait), in the order of the line.
constexpr int kWorkers = 512;    // workgroups that the line is cut for: two on every CU
constexpr int kOverhead = 4;     // units of a tile besides its steps
constexpr int kLeast = 8;        // units of a workgroup at least

template <typename T, int NP>
__global__ void __launch_bounds__(kAttnWaves* kWave, (Wave<T, NP>::OT <= 10 ? 2 : 1)) k_attn(AttnArgs a, uint32_t* tickets, float* parts) {
  using W = Wave<T, NP>;
  constexpr int kDims = NP * kRowPiece / static_cast<int>(sizeof(T));
  constexpr int NT = kAttnWaves * kWave;
  __shared__ Joined<kDims> sh;
  __shared__ int64_t sums[kAttnWaves];
  __shared__ int64_t where[2];
  __shared__ int32_t is_last;
  const int tid = threadIdx.x;
  const int lane = tid % kWave;
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c = lane % 16, g = lane / 16;
  const int per_slot = a.c.heads * a.tiles;
  auto steps_of = [&](Seen w) __attribute__((always_inline)) {
    const int blocks = w.none() ? 0 : (w.hi + kBlockTokens - 1) / kBlockTokens - w.lo / kBlockTokens;
    return (blocks + W::SB - 1) / W::SB;
  };
  auto cost_of = [&](int s) __attribute__((always_inline)) {
    return s < a.c.n_slots ? static_cast<int64_t>(per_slot) * (kOverhead + steps_of(seen_of(a, s))) : int64_t{0};
  };
  auto block_sum = [&](int64_t v, int64_t& before) __attribute__((always_inline)) {   // -> all; before: of lower threads
    int64_t upto = v;
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
      const int64_t o = __shfl_up(upto, m, kWave);
      if (lane >= m) upto += o;
    }
    __syncthreads();
    if (lane == kWave - 1) sums[wv] = upto;
    __syncthreads();
    int64_t all = 0;
    before = upto - v;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      before += w < wv ? sums[w] : 0;
      all += sums[w];
    }
    return all;
  };

  // the line's length, and the slot in which this workgroup's piece of it begins
  const int64_t first_cost = cost_of(tid);
  int64_t mine = first_cost;
  for (int s = tid + NT; s < a.c.n_slots; s += NT) mine += cost_of(s);
  int64_t before;
  const int64_t total = block_sum(mine, before);
  int64_t each = (total + kWorkers - 1) / kWorkers;
  if (each < kLeast) each = kLeast;
  const int64_t from = each * blockIdx.x;
  if (from >= total) return;
  const int64_t to = from + each < total ? from + each : total;
  int64_t passed = 0;
  for (int s0 = 0;; s0 += NT) {   // (ends: from < total)
    const int64_t cost = s0 == 0 ? first_cost : cost_of(s0 + tid);
    const int64_t all = block_sum(cost, before);
    if (from >= passed + before && from < passed + before + cost) {
      where[0] = s0 + tid;
      where[1] = passed + before;
    }
    passed += all;
    if (passed > from) break;
  }
  __syncthreads();
  int slot = __builtin_amdgcn_readfirstlane(static_cast<int>(where[0]));
  int64_t slot_at = where[1];
  uint32_t bad = 0;
  Seen seen = seen_of(a, slot);
  int steps = steps_of(seen);
  int64_t k = (from - slot_at) / (kOverhead + steps);   // head and tile of it
  for (;;) {
    const int64_t at = slot_at + k * (kOverhead + steps);
    if (at >= to) break;
    const int head = __builtin_amdgcn_readfirstlane(static_cast<int>(k) / a.tiles);
    const int tile = __builtin_amdgcn_readfirstlane(static_cast<int>(k) % a.tiles);
    const int queries = a.group - tile * 16 < 16 ? a.group - tile * 16 : 16;
    const int q0 = head * a.group + tile * 16;
    // this workgroup's steps of the tile
    const int64_t step0 = at + kOverhead;
    const int lo = __builtin_amdgcn_readfirstlane(from > step0 ? static_cast<int>(from - step0) : 0);
    const int hi = __builtin_amdgcn_readfirstlane(to - step0 < steps ? static_cast<int>(to - step0) : steps);
    if (steps == 0 && at >= from) {
      for (int i = tid; i < queries * a.c.head_dim / 4; i += NT)
        store4<T>(a.out, (static_cast<int64_t>(slot) * a.q_heads + q0) * a.c.head_dim + i * 4,
                  floatx4{0.f, 0.f, 0.f, 0.f});
      if (a.lse != nullptr && tid < queries)
        a.lse[static_cast<int64_t>(slot) * a.q_heads + q0 + tid] = -__builtin_inff();
    }
    if (lo < hi) {
      W w;
      w.clear();
      load_queries<T, NP>(a, w, slot, head, tile);
      walk<T, NP>(a, w, slot, head, seen, lo + wv, hi, kAttnWaves, bad);
      const float l = sum_of_groups(w.l);
      __syncthreads();   // the tile before this one has left LDS
      if (g == 0) {
        sh.m[wv][c] = w.m;
        sh.l[wv][c] = l;
      }
#pragma unroll
      for (int t = 0; t < W::OT; ++t) *reinterpret_cast<floatx4*>(&sh.o[wv][c][16 * t + 4 * g]) = w.o[t];
      __syncthreads();
      if (lo == 0 && hi == steps) {
        finish<T, kDims>(a, sh, slot, q0, queries, nullptr);
      } else {
        // a workgroup has two parts at most: of a tile that began before its piece
        // of the line, and of one that goes on behind it
        const int64_t floats = part_floats(a.group, kDims);
        finish<T, kDims>(a, sh, slot, q0, queries, parts + (2 * static_cast<int64_t>(blockIdx.x) + (lo == 0)) * floats);
        const int w0 = static_cast<int>(step0 / each), w1 = static_cast<int>((step0 + steps - 1) / each);
        wait_vmcnt<0>();
        __syncthreads();
        if (tid == 0)
          is_last = __hip_atomic_fetch_add(&tickets[w1], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                    static_cast<uint32_t>(w1 - w0);
        __syncthreads();
        if (is_last) {
          collect<kDims>(a, sh, queries, w1 - w0 + 1, [&](int p) __attribute__((always_inline)) {
            return parts + (2 * static_cast<int64_t>(w0 + p) + (p == 0)) * floats;
          });
          __syncthreads();
          finish<T, kDims>(a, sh, slot, q0, queries, nullptr);
          if (tid == 0) __hip_atomic_store(&tickets[w1], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
      }
    }
    if (++k == per_slot) {
      slot_at += static_cast<int64_t>(per_slot) * (kOverhead + steps);
      if (slot_at >= to) break;
      ++slot;
      seen = seen_of(a, slot);
      steps = steps_of(seen);
      k = 0;
    }
  }
  if (bad != 0 && a.flags != nullptr) atomicOr(a.flags, bad);
}

template <typename T, int NP>
hipError_t launch(const AttnArgs& a, void* workspace, hipStream_t st) {
  // no more workgroups than the longest line would have pieces
  constexpr int SB = Wave<T, NP>::SB;
  const int64_t longest = kOverhead + 1 + (static_cast<int64_t>(a.c.max_pages) * a.c.page / kBlockTokens + SB) / SB;
  const int64_t pieces = (longest * a.c.n_slots * a.c.heads * a.tiles + kLeast - 1) / kLeast;
  uint32_t* tickets = static_cast<uint32_t*>(workspace);
  float* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + align_up(kWorkers * sizeof(uint32_t), kAlign));
  k_attn<T, NP><<<static_cast<unsigned>(pieces < kWorkers ? pieces : kWorkers), kAttnWaves * kWave, 0, st>>>(
      a, tickets, parts);
  return hipGetLastError();
}

}  // namespace

static_assert(kWorkers * sizeof(uint32_t) <= FM_ATTN_TICKET_BYTES, "tickets");
size_t attn_ticket_bytes() { return align_up(kWorkers * sizeof(uint32_t), kAlign); }

size_t attn_workspace_bytes(const fm_kv_cache& c, int32_t q_heads) {
  const int dims = kv_pieces(c.head_dim, c.dtype) * kRowPiece / (c.dtype == FM_BF16 ? 2 : 4);
  const size_t floats = static_cast<size_t>(2 * kWorkers) * static_cast<size_t>(part_floats(q_heads / c.heads, dims));
  return attn_ticket_bytes() + align_up(floats * sizeof(float), kAlign);
}

hipError_t launch_attn(const AttnArgs& a, fm_dtype dt, void* workspace, hipStream_t st) {
  if (dt == FM_BF16) {
    switch (a.c.pieces) {
      case 1: return launch<uint16_t, 1>(a, workspace, st);
      case 2: return launch<uint16_t, 2>(a, workspace, st);
      case 3: return launch<uint16_t, 3>(a, workspace, st);
      case 4: return launch<uint16_t, 4>(a, workspace, st);
      case 5: return launch<uint16_t, 5>(a, workspace, st);
      case 6: return launch<uint16_t, 6>(a, workspace, st);
      case 7: return launch<uint16_t, 7>(a, workspace, st);
      case 8: return launch<uint16_t, 8>(a, workspace, st);
      default: return hipErrorInvalidValue;
    }
  }
  switch (a.c.pieces) {
    case 1: return launch<float, 1>(a, workspace, st);
    case 2: return launch<float, 2>(a, workspace, st);
    case 3: return launch<float, 3>(a, workspace, st);
    case 4: return launch<float, 4>(a, workspace, st);
    case 5: return launch<float, 5>(a, workspace, st);
    case 6: return launch<float, 6>(a, workspace, st);
    case 7: return launch<float, 7>(a, workspace, st);
    case 8: return launch<float, 8>(a, workspace, st);
    case 9: return launch<float, 9>(a, workspace, st);
    case 10: return launch<float, 10>(a, workspace, st);
    case 11: return launch<float, 11>(a, workspace, st);
    case 12: return launch<float, 12>(a, workspace, st);
    case 13: return launch<float, 13>(a, workspace, st);
    case 14: return launch<float, 14>(a, workspace, st);
    case 15: return launch<float, 15>(a, workspace, st);
    case 16: return launch<float, 16>(a, workspace, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace fm
